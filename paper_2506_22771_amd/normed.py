"""Dense Forward-Forward stacks with a learned layer norm in front of every layer, trained in one pass per set.

    a -> layer norm (gamma_i, beta_i) -> int8 layer W_i -> u_i = W_i y -> ReLU -> next layer;  goodness G_i = ||relu(u_i)||^2

A layer that sees its input at its full length can read the goodness of the layer below off that length; a norm in between takes it away.
The forward pass is the library's int8 one (quantise, contraction, goodness, loss derivative).  What the updates need once the goodness of every layer is
known is kept in 8 bits: the checkpoint of the normalised input h_i, which the norm writes as it goes, and that of u_i; int32 accumulators, layer
inputs and the norms' outputs are scratch.  Then, per set and from the last layer down, with c_i = dL_i/dG_i and E_k = 0 (Eq. (4) as an exact derivative):

    g_i = (2 c_i relu(u_i) + lambda E_i) relu'(u_i)    what layer i learns from:   dW_i from g_i and the checkpoint of h_i,
                                                        dgamma_i, dbeta_i from g_i W_i through the norm
    t_i = (2 c_i relu(u_i) + E_i) relu'(u_i)           what the layers below get:  E_{i-1} = dx of the norm at t_i W_i

lambda = 0 is the layer-local rule: nothing is handed down.  The products with W_i run in int8, as every product of the method.

    python -m paper_2506_22771_amd.normed      trains a small stack on synthetic two-set data and prints its losses"""
from __future__ import annotations

import dataclasses
import math
from typing import List, Optional, Sequence

import torch

from . import binding as ff


# Stochastic-rounding streams of this path (no stack here has the gradients of FF_LOOKAHEAD_CHAIN, whose number the first takes).
KIND_KEPT, KIND_DOWN = ff.KIND_CHAIN, 3


@dataclasses.dataclass
class _Dense:   # what layer_desc asks for
    in_features: int
    out_features: int
    kind: str = "dense"
    H: int = 0
    W: int = 0
    C_in: int = 0
    C_out: int = 0
    ksize: int = 0
    stride: int = 0
    pad: int = 0
    relu: int = 1
    l2norm_out: int = 0


@dataclasses.dataclass
class Kept:
    """What one layer keeps of one pass until its update."""
    h: tuple            # checkpoint of the normalised input: codes, exponent bytes
    u: tuple            # checkpoint of the activation's argument
    rstd: torch.Tensor
    goodness: torch.Tensor
    coeff: torch.Tensor
    loss: torch.Tensor

    def bytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (*self.h, *self.u, self.rstd, self.goodness, self.coeff))


@dataclasses.dataclass
class Gradients:
    weight: List[torch.Tensor]
    gamma: List[torch.Tensor]
    beta: List[torch.Tensor]


class NormedNet:
    """widths: features of the input and of every layer.  Parameters are fp32 on the device; w[i] is [widths[i+1], widths[i]]."""

    def __init__(self, widths: Sequence[int], batch: int, theta: float = 2.0, eps: float = 1e-5, seed: int = 0, device="cuda"):
        self.widths, self.batch, self.theta, self.eps, self.seed = list(widths), batch, theta, eps, seed
        self.k = len(widths) - 1
        g = torch.Generator(device="cpu").manual_seed(seed)
        new = lambda *shape, of=torch.float32: torch.zeros(shape, dtype=of, device=device)  # noqa: E731
        self.w, self.gamma, self.beta, self.w_q, self.w_qt, self.s_w, self.desc = [], [], [], [], [], [], []
        for K, N in zip(self.widths, self.widths[1:]):
            bound = math.sqrt(6.0 / K)
            self.w.append(((torch.rand((N, K), generator=g) * 2 - 1) * bound).to(device))
            self.gamma.append(torch.ones(K, device=device))
            self.beta.append(new(K))
            self.w_q.append(new(N, ff.ff_pitch(K), of=torch.int8))
            self.w_qt.append(new(K, ff.ff_pitch(N), of=torch.int8))
            self.s_w.append(new(1))
            self.desc.append(ff.layer_desc(_Dense(K, N), batch))
        self.grad = Gradients([new(*w.shape) for w in self.w], [new(K) for K in self.widths[:-1]], [new(K) for K in self.widths[:-1]])
        need = max([ff.WS_MIN_BYTES] + [max(ff.ff_layer_norm_workspace_bytes(batch, K), ff.ff_ckpt_weight_grad_workspace_bytes(batch, N, K),
                                            ff.ff_layer_workspace_bytes(d)) for K, N, d in zip(self.widths, self.widths[1:], self.desc)])
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        self._requantise()

    def _requantise(self) -> None:
        for i, w in enumerate(self.w):
            ff.ff_quantize(w, w.shape[0], w.shape[1], ff.ROUND_NEAREST, 0, 0, self.w_q[i], self.w_qt[i], self.s_w[i], self.ws)

    def forward(self, x: torch.Tensor, sign: int, step: int = 0) -> List[Kept]:
        """One set through all layers; sign: ff.PASS_POS or ff.PASS_NEG."""
        B, kept, a, p = self.batch, [], x, int(sign == ff.PASS_NEG)
        new = lambda *shape, of=torch.float32: torch.empty(shape, dtype=of, device=x.device)  # noqa: E731
        for i in range(self.k):
            K, N = self.widths[i], self.widths[i + 1]
            y, mean, rstd, h = new(B, K), new(B), new(B), ff.ckpt_empty(B, K, x.device)
            ff.ff_layer_norm_forward(a, self.gamma[i], self.beta[i], self.eps, y, mean, rstd, *h, ff.ROUND_STOCHASTIC, self.seed,
                                     ff.ff_stream_tag(step, i, p, KIND_KEPT))
            a_q, s_a = new(B, ff.ff_pitch(K), of=torch.int8), new(1)
            ff.ff_quantize(y, B, K, ff.ROUND_STOCHASTIC, self.seed, ff.ff_stream_tag(step, i, p, ff.KIND_ACT), a_q, None, s_a, self.ws)
            acc, gsum, vmax = new(B, ff.ff_pitch32(N), of=torch.int32), new(B, of=torch.int64), new(B, of=torch.int32)
            ff.ff_layer_forward(self.desc[i], a_q, self.w_q[i], acc, gsum, vmax, self.ws)
            good, coeff, loss = new(B), new(B), new(1)
            ff.ff_goodness_loss(self.desc[i], gsum, vmax, s_a, self.s_w[i], sign, self.theta, good, coeff, loss, None)
            arg = acc[:, :N].float() * (s_a * self.s_w[i])
            u = ff.ckpt_empty(B, N, x.device)
            ff.ff_ckpt_store(arg, ff.ROUND_NEAREST, 0, 0, *u)
            kept.append(Kept(h, u, rstd, good, coeff, loss))
            a = arg.relu_()
        return kept

    def _through_weights(self, i: int, d: torch.Tensor, tag: int) -> torch.Tensor:
        """d W_i in int8: the gradient at the norm's output."""
        B, K, N = self.batch, self.widths[i], self.widths[i + 1]
        d_q, s_d = torch.empty((B, ff.ff_pitch(N)), dtype=torch.int8, device=d.device), torch.empty(1, device=d.device)
        ff.ff_quantize(d, B, N, ff.ROUND_STOCHASTIC, self.seed, tag, d_q, None, s_d, self.ws)
        e_acc = torch.empty((B, ff.ff_pitch32(K)), dtype=torch.int32, device=d.device)
        ff.ff_layer_input_grad(self.desc[i], d_q, self.w_qt[i], e_acc, self.ws)
        return e_acc[:, :K].float() * (s_d * self.s_w[i])

    def backward(self, kept: List[Kept], sign: int, lam: float, step: int = 0, accumulate: bool = False) -> Gradients:
        """Gradients of one set, summed over its samples, into self.grad (added to what is there with `accumulate`)."""
        p, down = int(sign == ff.PASS_NEG), None
        for i in reversed(range(self.k)):
            s, K, N = kept[i], self.widths[i], self.widths[i + 1]
            g = torch.empty((self.batch, N), device=s.coeff.device)
            ff.ff_ckpt_act_backward(*s.u, ff.ACT_RELU, s.coeff, None if down is None else down * lam, g)
            ff.ff_ckpt_weight_grad(g, *s.h, self.gamma[i], self.beta[i], self.grad.weight[i], None, accumulate, self.ws)
            dy = self._through_weights(i, g, ff.ff_stream_tag(step, i, p, ff.KIND_GRAD))
            grads = self.grad.gamma[i], self.grad.beta[i]
            below = None if lam == 0.0 or i == 0 else torch.empty((self.batch, K), device=dy.device)
            alike = down is None or lam == 1.0      # g is t as well: what the layers below get of the ones above is not scaled twice
            ff.ff_layer_norm_backward(dy, None, None, *s.h, s.rstd, self.gamma[i], below if alike else None, *grads, accumulate, self.ws)
            if below is not None and not alike:
                ff.ff_ckpt_act_backward(*s.u, ff.ACT_RELU, s.coeff, down, g)
                dy = self._through_weights(i, g, ff.ff_stream_tag(step, i, p, KIND_DOWN))
                ff.ff_layer_norm_backward(dy, None, None, *s.h, s.rstd, self.gamma[i], below, None, None, False, self.ws)
            down = below
        return self.grad

    def step(self, x_pos: torch.Tensor, x_neg: torch.Tensor, lam: float, lr: float, step: int = 0) -> torch.Tensor:
        """One update from both sets; returns the mean losses [layers, 2] (positive, negative)."""
        pos, neg = self.forward(x_pos, ff.PASS_POS, step), self.forward(x_neg, ff.PASS_NEG, step)
        self.backward(pos, ff.PASS_POS, lam, step)
        self.backward(neg, ff.PASS_NEG, lam, step, accumulate=True)
        rate = -lr / (2 * self.batch)
        for ps, gs in ((self.w, self.grad.weight), (self.gamma, self.grad.gamma), (self.beta, self.grad.beta)):
            for p, g in zip(ps, gs):
                p.add_(g, alpha=rate)
        self._requantise()
        return torch.stack([torch.cat([a.loss, b.loss]) for a, b in zip(pos, neg)])


def two_sets(batch: int, features: int, seed: int, device="cuda", classes: int = 10):
    """Synthetic samples with their class's pattern added, and one-hot labels in the first features: true (positive set) or wrong (negative set)."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    pattern = torch.rand((classes, features), generator=torch.Generator(device="cpu").manual_seed(7))
    label = torch.randint(classes, (batch,), generator=g)
    other = (label + torch.randint(1, classes, (batch,), generator=g)) % classes
    x = 0.5 * torch.rand((batch, features), generator=g) + pattern[label]
    sets = []
    for lab in (label, other):
        s = x.clone()
        s[:, :classes] = 3.0 * torch.nn.functional.one_hot(lab, classes)
        sets.append(s.to(device))
    return sets


def main(steps: int = 200, widths: Sequence[int] = (784, 500, 500), batch: int = 64, lam: float = 0.05, lr: float = 0.03,
         report: Optional[int] = 25) -> List[float]:
    net = NormedNet(widths, batch, theta=float(widths[1]) / 2)
    history = []
    for t in range(steps):
        loss = net.step(*two_sets(batch, widths[0], 1000 + t), lam, lr, t)
        if report and (t % report == 0 or t == steps - 1):
            history.append(float(loss.mean()))
            print(f"step {t:4d}: mean loss {history[-1]:.4f}, by layer (positive, negative) {[[round(v, 3) for v in r] for r in loss.tolist()]}", flush=True)
    return history


if __name__ == "__main__":
    main()
