"""Forward-Forward stacks over images: patch layers with group norm, then gated layers, dropout behind every one, trained in one pass per set.

    map layer     a -> patches of side x side pixels -> int8 layer W -> group norm (gamma, beta) -> SiLU
    gated layer   a -> layer norm (gamma, beta) -> int8 layer W, whose first half of outputs gates the second: SiLU(g) u

A layer's goodness is the sum of its squared activities, G; what the next one gets are those activities behind dropout.  Norms, gated layers and dropout take and give
their goodness and its derivative c = dL/dG themselves; what an update needs once every goodness is known is kept in 8 bits: the checkpoints of a map layer's
patches and of its normalised map, those of a gated layer's normalised input, of g and of u.  No mask is kept: the backward pass drops what the forward pass did
by the same random word.  Per set and from the last layer down, with c_i and E_k = 0 (Eq. (4) as an exact derivative, as in normed.py):

    layer i learns from 2 c_i f + lambda E_i,   the layers below get what 2 c_i f + E_i, through its norm and its weights, is at its input: E_{i-1}, behind dropout

    python -m paper_2506_22771_amd.gated      trains a small stack on synthetic two-set images and prints its losses"""
from __future__ import annotations

import dataclasses
import math
from typing import List, Optional, Sequence, Tuple

import torch

from . import binding as ff
from .normed import KIND_DOWN, KIND_KEPT, Gradients, _Dense

# Streams of random words of this path, beside those of normed.py.
KIND_DROP, KIND_INPUT = 4, 5


@dataclasses.dataclass
class Layer:
    gated: bool
    rows: int            # of the contraction: pixels, or samples
    k: int               # features of its input
    n: int               # its activities per row
    side: int = 1        # map layer: of a patch
    size: Tuple[int, int, int] = (0, 0, 0)   # and of the map it is cut from: height, width, channels
    groups: int = 1

    @property
    def out(self) -> int:
        return 2 * self.n if self.gated else self.n

    @property
    def normed(self) -> int:
        return self.k if self.gated else self.n


@dataclasses.dataclass
class Kept:
    """What one layer keeps of one pass until its update."""
    a: Optional[tuple]   # map layer: checkpoint of its patches
    h: tuple             # checkpoint of the norm's normalised values
    g: Optional[tuple]   # gated layer: checkpoints of its projections
    u: Optional[tuple]
    rstd: torch.Tensor
    goodness: torch.Tensor
    coeff: torch.Tensor
    loss: torch.Tensor


class GatedNet:
    """image: (height, width, channels); maps: (side of a patch, channels, groups) of every map layer; gated: activities of every gated layer.  Inputs are
    [batch, height * width, channels], fp32.  Parameters are fp32 on the device; w[i] is [outputs, inputs].  theta: goodness per activity."""

    def __init__(self, image: Tuple[int, int, int], maps: Sequence[Tuple[int, int, int]], gated: Sequence[int], batch: int, theta: float = 0.3,
                 p_drop: float = 0.1, eps: float = 1e-5, seed: int = 0, device="cuda"):
        self.batch, self.p_drop, self.eps, self.seed = batch, p_drop, eps, seed
        self.layers: List[Layer] = []
        H, W, C = image
        for side, n, groups in maps:
            if H % side or W % side:
                raise ValueError(f"patches of {side} x {side} pixels do not cover a map of {H} x {W}")
            self.layers.append(Layer(False, batch * (H // side) * (W // side), side * side * C, n, side, (H, W, C), groups))
            H, W, C = H // side, W // side, n
        k = H * W * C
        for n in gated:
            self.layers.append(Layer(True, batch, k, n))
            k = n
        gen = torch.Generator(device="cpu").manual_seed(seed)
        new = lambda *shape, of=torch.float32: torch.zeros(shape, dtype=of, device=device)  # noqa: E731
        self.w, self.gamma, self.beta, self.w_q, self.w_qt, self.s_w, self.desc, self.theta = [], [], [], [], [], [], [], []
        need = ff.WS_MIN_BYTES
        for y in self.layers:
            self.w.append(((torch.rand((y.out, y.k), generator=gen) * 2 - 1) * math.sqrt(6.0 / y.k)).to(device))
            self.gamma.append(torch.ones(y.normed, device=device))
            self.beta.append(new(y.normed))
            self.w_q.append(new(y.out, ff.ff_pitch(y.k), of=torch.int8))
            self.w_qt.append(new(y.k, ff.ff_pitch(y.out), of=torch.int8))
            self.s_w.append(new(1))
            self.desc.append(ff.layer_desc(_Dense(y.k, y.out), y.rows))
            self.theta.append(theta * (y.rows // batch * y.n))
            norm = ff.ff_layer_norm_workspace_bytes(batch, y.k) if y.gated else ff.ff_group_norm_workspace_bytes(batch, y.rows // batch, y.n, y.groups)
            need = max(need, norm, ff.ff_gated_workspace_bytes(batch, y.n, y.k) if y.gated else 0, ff.ff_layer_workspace_bytes(self.desc[-1]),
                       ff.ff_ckpt_weight_grad_workspace_bytes(y.rows, y.out, y.k))
        self.grad = Gradients([new(*w.shape) for w in self.w], [new(*g.shape) for g in self.gamma], [new(*b.shape) for b in self.beta])
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        self._requantise()

    def _requantise(self) -> None:
        for i, w in enumerate(self.w):
            ff.ff_quantize(w, w.shape[0], w.shape[1], ff.ROUND_NEAREST, 0, 0, self.w_q[i], self.w_qt[i], self.s_w[i], self.ws)

    def _patches(self, y: Layer, a: torch.Tensor) -> torch.Tensor:
        (H, W, C), s = y.size, y.side
        return a.reshape(self.batch, H // s, s, W // s, s, C).permute(0, 1, 3, 2, 4, 5).reshape(y.rows, y.k)

    def _pixels(self, y: Layer, e: torch.Tensor) -> torch.Tensor:
        """Of patches, their map's rows."""
        (H, W, C), s = y.size, y.side
        return e.reshape(self.batch, H // s, W // s, s, s, C).permute(0, 1, 3, 2, 4, 5).reshape(self.batch * H * W, C)

    def forward(self, x: torch.Tensor, sign: int, step: int = 0, step_dev: Optional[torch.Tensor] = None) -> List[Kept]:
        """One set through all layers; sign: ff.PASS_POS or ff.PASS_NEG.  step_dev: a step on the device that dropout adds to `step` (for graphs)."""
        B, kept, a, p = self.batch, [], x, int(sign == ff.PASS_NEG)
        new = lambda *shape, of=torch.float32: torch.empty(shape, dtype=of, device=x.device)  # noqa: E731
        for i, y in enumerate(self.layers):
            tag = lambda kind: ff.ff_stream_tag(step, i, p, kind)  # noqa: B023,E731
            a = a.reshape(B, y.k) if y.gated else self._patches(y, a)
            codes, good = ff.ckpt_empty(y.rows, y.normed, x.device), new(B)
            if y.gated:
                normal, mean, rstd = new(B, y.k), new(B), new(B)
                ff.ff_layer_norm_forward(a, self.gamma[i], self.beta[i], self.eps, normal, mean, rstd, *codes, ff.ROUND_STOCHASTIC, self.seed, tag(KIND_KEPT))
                a = normal
            a_q, s_a = new(y.rows, ff.ff_pitch(y.k), of=torch.int8), new(1)
            ff.ff_quantize(a, y.rows, y.k, ff.ROUND_STOCHASTIC, self.seed, tag(ff.KIND_ACT), a_q, None, s_a, self.ws)
            out = new(y.rows, y.n)
            if y.gated:
                g, u, patches = ff.ckpt_empty(B, y.n, x.device), ff.ckpt_empty(B, y.n, x.device), None
                ff.ff_gated_forward(a_q, self.w_q[i], s_a, self.s_w[i], y.k, ff.ACT_SILU, out, good, *g, *u, self.ws)
            else:
                g, u, patches = None, None, ff.ckpt_empty(y.rows, y.k, x.device)
                ff.ff_ckpt_store(a, ff.ROUND_STOCHASTIC, self.seed, tag(KIND_INPUT), *patches)
                acc, gsum, vmax = new(y.rows, ff.ff_pitch32(y.n), of=torch.int32), new(y.rows, of=torch.int64), new(y.rows, of=torch.int32)
                ff.ff_layer_forward(self.desc[i], a_q, self.w_q[i], acc, gsum, vmax, self.ws)
                arg, mean, rstd = acc[:, :y.n].float() * (s_a * self.s_w[i]), new(B, y.groups), new(B, y.groups)
                ff.ff_group_norm_forward(arg, B, y.groups, self.gamma[i], self.beta[i], self.eps, ff.ACT_SILU, out, mean, rstd, good, *codes,
                                         ff.ROUND_STOCHASTIC, self.seed, tag(KIND_KEPT), self.ws)
            far = float(1 if sign == ff.PASS_POS else -1) * (good - self.theta[i])
            coeff = torch.sigmoid(-far) * (-1.0 if sign == ff.PASS_POS else 1.0)
            kept.append(Kept(patches, codes, g, u, rstd, good, coeff, torch.nn.functional.softplus(-far).mean().reshape(1)))
            a = torch.empty_like(out)
            ff.ff_dropout(out, None, self.p_drop, self.seed, tag(KIND_DROP), step_dev, a)
        return kept

    def _through_weights(self, i: int, d: torch.Tensor, tag: int) -> torch.Tensor:
        """d W_i in int8: the gradient at the contraction's input."""
        y = self.layers[i]
        d_q, s_d = torch.empty((y.rows, ff.ff_pitch(y.out)), dtype=torch.int8, device=d.device), torch.empty(1, device=d.device)
        ff.ff_quantize(d, y.rows, y.out, ff.ROUND_STOCHASTIC, self.seed, tag, d_q, None, s_d, self.ws)
        e_acc = torch.empty((y.rows, ff.ff_pitch32(y.k)), dtype=torch.int32, device=d.device)
        ff.ff_layer_input_grad(self.desc[i], d_q, self.w_qt[i], e_acc, self.ws)
        return e_acc[:, :y.k].float() * (s_d * self.s_w[i])

    def _layer_backward(self, i: int, s: Kept, dy: Optional[torch.Tensor], tag: int, grads: bool, below: bool, accumulate: bool) -> Optional[torch.Tensor]:
        """Through one layer, from 2 c f + dy: its parameters' gradients into self.grad, or the gradient at its input, or both."""
        y = self.layers[i]
        dw, dgamma, dbeta = (self.grad.weight[i], self.grad.gamma[i], self.grad.beta[i]) if grads else (None, None, None)
        d = torch.empty((y.rows, y.out), device=s.coeff.device)
        if not y.gated:
            ff.ff_group_norm_backward(dy, s.coeff, None, None, *s.h, s.rstd, self.batch, y.groups, self.gamma[i], self.beta[i], ff.ACT_SILU, d,
                                      dgamma, dbeta, accumulate, self.ws)
            if grads:
                ff.ff_ckpt_weight_grad(d, *s.a, None, None, dw, None, accumulate, self.ws)
            return self._pixels(y, self._through_weights(i, d, tag)) if below else None
        ff.ff_gated_backward(*s.g, *s.u, ff.ACT_SILU, s.coeff, dy, d[:, :y.n], d[:, y.n:])
        if grads:
            ff.ff_ckpt_weight_grad(d, *s.h, self.gamma[i], self.beta[i], dw, None, accumulate, self.ws)
        e = torch.empty((y.rows, y.k), device=d.device) if below else None
        ff.ff_layer_norm_backward(self._through_weights(i, d, tag), None, None, *s.h, s.rstd, self.gamma[i], e, dgamma, dbeta, accumulate, self.ws)
        return e

    def backward(self, kept: List[Kept], sign: int, lam: float, step: int = 0, accumulate: bool = False, step_dev: Optional[torch.Tensor] = None) -> Gradients:
        """Gradients of one set, summed over its samples, into self.grad (added to what is there with `accumulate`)."""
        p, down = int(sign == ff.PASS_NEG), None
        for i in reversed(range(len(self.layers))):
            y, s = self.layers[i], kept[i]
            if down is not None:   # what was dropped of this layer's activities had no part in what the layers above learnt
                dropped = down.reshape(y.rows, y.n)
                down = torch.empty_like(dropped)
                ff.ff_dropout(dropped, None, self.p_drop, self.seed, ff.ff_stream_tag(step, i, p, KIND_DROP), step_dev, down)
            more = lam != 0.0 and i > 0
            alike = down is None or lam == 1.0   # what this layer learns from is what the layers below get
            below = self._layer_backward(i, s, None if down is None else down if alike else down * lam, ff.ff_stream_tag(step, i, p, ff.KIND_GRAD),
                                         True, more and alike, accumulate)
            if more and not alike:
                below = self._layer_backward(i, s, down, ff.ff_stream_tag(step, i, p, KIND_DOWN), False, True, False)
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


def two_sets(batch: int, image: Tuple[int, int, int], seed: int, device="cuda", classes: int = 10) -> List[torch.Tensor]:
    """Synthetic images with their class's pattern added, and one-hot labels in their first pixels: true (positive set) or wrong (negative set)."""
    H, W, C = image
    g = torch.Generator(device="cpu").manual_seed(seed)
    pattern = torch.rand((classes, H * W, C), generator=torch.Generator(device="cpu").manual_seed(7))
    label = torch.randint(classes, (batch,), generator=g)
    other = (label + torch.randint(1, classes, (batch,), generator=g)) % classes
    x = 0.5 * torch.rand((batch, H * W, C), generator=g) + pattern[label]
    sets = []
    for lab in (label, other):
        s = x.clone()
        s[:, :classes] = 3.0 * torch.nn.functional.one_hot(lab, classes)[:, :, None]
        sets.append(s.to(device))
    return sets


def main(steps: int = 200, image: Tuple[int, int, int] = (32, 32, 3), batch: int = 64, lam: float = 0.05, lr: float = 3e-4, report: Optional[int] = 25) -> List[float]:
    net = GatedNet(image, ((4, 64, 8), (2, 128, 16)), (256, 256), batch)
    history = []
    for t in range(steps):
        loss = net.step(*two_sets(batch, image, 1000 + t), lam, lr, t)
        if report and (t % report == 0 or t == steps - 1):
            history.append(float(loss.mean()))
            print(f"step {t:4d}: mean loss {history[-1]:.4f}, by layer (positive, negative) {[[round(v, 3) for v in r] for r in loss.tolist()]}", flush=True)
    return history


if __name__ == "__main__":
    main()
