"""Stacks with learned norms, trained from 8-bit checkpoints: the five operations together."""
import numpy as np
import pytest
import torch

import paper_2506_22771_amd as ff
from norm_util import U, split_ckpt, values, within
from oracle import norm_oracle as N

pytestmark = pytest.mark.gpu


@pytest.fixture()
def small():
    from paper_2506_22771_amd.normed import NormedNet, two_sets
    net = NormedNet((100, 70, 44, 30), 48, theta=4.0, seed=3)
    g = torch.Generator("cuda").manual_seed(1)
    for w, ga, be in zip(net.w, net.gamma, net.beta):    # goodness of a few units, where the loss derivatives are smooth; norms that do something
        w.mul_(0.25)
        ga.add_(0.3 * torch.randn(ga.shape, generator=g, device="cuda"))
        be.add_(0.3 * torch.randn(be.shape, generator=g, device="cuda"))
    net._requantise()
    return net, two_sets(48, 100, 5)


def kept_values(s, K, n):
    return N.ckpt_load(*split_ckpt(*s.h, K)), N.ckpt_load(*split_ckpt(*s.u, n))


def test_top_layer_gradients_are_those_of_what_was_kept(small):
    """The last layer's weight gradient has no 8-bit gradient in it: fp32's roundings alone separate it from 64 bits."""
    net, (xp, _) = small
    kept = net.forward(xp, ff.PASS_POS)
    grad = net.backward(kept, ff.PASS_POS, 0.3)
    h, u = kept_values(kept[-1], 44, 30)
    c = values(kept[-1].coeff)
    g = N.act_backward("relu", u, c, None)
    dw, _ = N.weight_grad(g, h, values(net.gamma[-1]), values(net.beta[-1]))
    size = np.abs(g).T @ np.abs(h) * np.abs(values(net.gamma[-1])) + np.abs(g).sum(0)[:, None] * np.abs(values(net.beta[-1]))
    within(values(grad.weight[-1]), dw, (48 + 12) * U * size, "dw")
    # the norm's gradients pass the int8 product: half a step of the quantised gradient per element at random, 1 % of a row's sum at most
    dy = g @ values(net.w[-1])
    _, dg, db = N.norm_backward(dy, h, np.ones(48), None)
    for got, ref in ((grad.gamma[-1], dg), (grad.beta[-1], db)):
        assert np.linalg.norm(values(got) - ref) < 0.05 * np.linalg.norm(ref)


@pytest.mark.parametrize("lam", [0.0, 0.3, 1.0])
def test_gradients_against_the_model_in_64_bits(small, lam):
    """dL_new of every parameter, L_new = L_i + lambda (L_{i+1} + ...), of the unquantised model.  8-bit steps of inputs (0.9 % of their size), weights
    (0.4 %), kept activities (0.6 %) and gradients (1.5 %) add up to 2 % a layer, and to 6 % over three.  ReLU passes a unit or not: which ones, the int8
    forward decides (1 % of the units differ, those next to zero, and their gradients whole), so the model takes that from what was kept."""
    net, sets = small
    passes = []
    for sign, x in ((ff.PASS_POS, sets[0]), (ff.PASS_NEG, sets[1])):
        kept = net.forward(x, sign)
        net.backward(kept, sign, lam, accumulate=sign == ff.PASS_NEG)
        passes.append([torch.from_numpy((kept_values(s, K, n)[1] > 0).astype(np.float64)) for s, K, n in zip(kept, net.widths, net.widths[1:])])
    P = [[t.double().cpu().requires_grad_() for t in ts] for ts in (net.w, net.gamma, net.beta)]
    losses = []
    for sign, x, on in ((1, sets[0], passes[0]), (-1, sets[1], passes[1])):
        a, per = x.double().cpu(), []
        for w, ga, be, passed in zip(*P, on):
            y = torch.nn.functional.layer_norm(a, (a.shape[1],), ga, be, net.eps)
            a = (y @ w.t()) * passed
            per.append(torch.nn.functional.softplus(-sign * ((a * a).sum(1) - net.theta)).sum())
        losses.append(per)
    for i in range(3):
        total = sum(p[i] + lam * sum(p[i + 1:]) for p in losses)
        want = torch.autograd.grad(total, [ts[i] for ts in P], retain_graph=True)
        for got, ref, what in zip((net.grad.weight[i], net.grad.gamma[i], net.grad.beta[i]), want, ("weight", "gamma", "beta")):
            err = (got.double().cpu() - ref).norm() / ref.norm()
            assert err < 0.06, (i, what, float(err))


def test_without_lookahead_a_layer_learns_as_if_it_were_the_last(small):
    from paper_2506_22771_amd.normed import NormedNet
    net, (xp, _) = small
    one = NormedNet((100, 70), 48, theta=4.0, seed=3)
    for a, b in ((one.w[0], net.w[0]), (one.gamma[0], net.gamma[0]), (one.beta[0], net.beta[0])):
        a.copy_(b)
    one._requantise()
    a, b = net.backward(net.forward(xp, ff.PASS_POS), ff.PASS_POS, 0.0), one.backward(one.forward(xp, ff.PASS_POS), ff.PASS_POS, 0.0)
    assert torch.equal(a.weight[0], b.weight[0]) and torch.equal(a.gamma[0], b.gamma[0]) and torch.equal(a.beta[0], b.beta[0])


def test_what_is_kept_is_a_byte_a_value(small):
    net, (xp, _) = small
    for s, K, n in zip(net.forward(xp, ff.PASS_POS), net.widths, net.widths[1:]):
        padded = 48 * (ff.ff_pitch(K) + ff.ff_pitch(ff.ff_ckpt_blocks(K)) + ff.ff_pitch(n) + ff.ff_pitch(ff.ff_ckpt_blocks(n)))
        assert s.bytes() == padded + 3 * 4 * 48


def test_training_lowers_the_loss_and_is_reproducible():
    from paper_2506_22771_amd.normed import NormedNet, two_sets
    ends = []
    for _ in range(2):
        net = NormedNet((200, 128, 96), 64, theta=64.0, seed=0)
        losses = [float(net.step(*two_sets(64, 200, t), 0.05, 0.03, t).mean()) for t in range(120)]
        assert np.mean(losses[-10:]) < 0.8 * np.mean(losses[:10])
        ends.append(torch.cat([t.reshape(-1) for t in (*net.w, *net.gamma, *net.beta)]))
    assert torch.equal(*ends)
