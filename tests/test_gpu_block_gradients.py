"""The block's training gradients against the fp64 chain (layer oracle, then the norm's formula), and against differences of
its own forward along directions in which a wrong gradient cannot hide.

Bars.  The layer's own: max |a - b| <= 2e-2 max |b| for BF16 (`E` below for the gradient that enters the norm).  Through the
norm an error of that size becomes at most rstd (|w| E + |xhat| mean(|w xhat|) E), and dx is rounded once (2^-8).  Each bar
is also held against the oracle with a mistake planted in it, which has to miss it clearly: a bar that every gradient
passes is none."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import block_ops as Q
from paper_2604_23108_b200 import binding as B
from paper_2604_23108_b200.block import MoeBlock

from _util import max_rel

BF16_BAR = 2e-2
np64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
D, WIDTHS, N, KG, KE = 256, (128, 264, 72), 4, 2, 3


def tensors(T, seed=0):
    """x, residual, dy, dh, norm weight, router, w13, w2 in BF16 on the CPU."""
    g = torch.Generator().manual_seed(seed)
    n = lambda s, *sh: (torch.randn(*sh, generator=g) * s).bfloat16()  # noqa: E731
    return ([n(1, T, D) for _ in range(4)] + [(1 + 0.1 * torch.randn(D, generator=g)).bfloat16(), n(0.1, len(WIDTHS) * (1 + N), D),
            [n(0.06, N, 2 * w, D) for w in WIDTHS], [n(0.06, N, D, w) for w in WIDTHS]])


def chain(u, logits, h, rstd, dy, dh, norm_w, w_r, w13, w2, mistake=None):
    """(dx, dnorm, layer's gradients, bound on dx) in fp64 from what the forward left."""
    cfg = O.OracleConfig(d_model=D, n_groups=len(WIDTHS), experts_per_group=N, k_groups=KG, k_experts=KE, group_width=list(WIDTHS))
    fwd = O.layer_forward(cfg, u, w_r, w13, w2, logits=logits, mode="spec")
    bwd = O.layer_backward(fwd, w13, w2, dy, with_aux=True)
    du = {None: bwd["dx"], "no router": bwd["dx_experts"], "no experts": bwd["dx_router"],
          "sign of the layer": -bwd["dx"]}.get(mistake, bwd["dx"])
    dx, dnorm = Q.norm_bwd(du, None if mistake == "no dh" else dh, h, norm_w, rstd)
    if mistake == "no norm":
        dx = du + dh
    elif mistake == "sign":
        dx = -dx
    rs, xh, E = rstd[:, None], np.abs(h * rstd[:, None]), BF16_BAR * np.max(np.abs(bwd["dx"]))
    bound = rs * E * (np.abs(norm_w) + xh * np.mean(np.abs(norm_w) * xh, axis=1, keepdims=True)) + 2.0 ** -8 * np.abs(dx)
    return dx, dnorm, bwd, bound


MISTAKES = ["no router", "no experts", "sign of the layer", "no dh", "no norm", "sign"]


def planted(good, args):
    """Each mistake misses the bar on dx, or (where dx carries little of it) the bar on dnorm, by more than half."""
    dx, dnorm, _, bound = good
    for m in MISTAKES:
        bad = chain(*args, mistake=m)
        assert np.max(np.abs(bad[0] - dx) / bound) > 1.5 or max_rel(bad[1], dnorm) > 1.5 * BF16_BAR, m


def test_planted_mistakes_are_seen():
    x, r, dy, dh, nw, w_r, w13, w2 = tensors(60)
    h, u, rstd = Q.norm_fwd(np64(x), np64(r), np64(nw), 1e-6)
    w_r, w13, w2 = np64(w_r), [np64(w) for w in w13], [np64(w) for w in w2]
    logits = O.router_logits(u, w_r).astype(np.float32).astype(np.float64)
    args = (u, logits, h, rstd, np64(dy), np64(dh), np64(nw), w_r, w13, w2)
    planted(chain(*args), args)


def make(T, seed):
    cpu = tensors(T, seed)
    x, r, dy, dh, nw, w_r = (t.cuda() for t in cpu[:6])
    cfg = B.Config(D, len(WIDTHS), N, KG, KE, list(WIDTHS))
    return MoeBlock(cfg, nw, w_r, [w.cuda() for w in cpu[6]], [w.cuda() for w in cpu[7]]), x, r, dy, dh


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 60, 333])
@pytest.mark.parametrize("with_dh", [True, False])
def test_training_step_against_the_fp64_chain(T, with_dh):
    block, x, r, dy, dh = make(T, seed=T)
    dh = dh if with_dh else None
    block.train_forward(x, r)
    dx = block.train_backward(dy, dh)
    b, g = block._buffers("train", T), block.grads(T)
    w_r, w13, w2 = np64(block.w_router), [np64(w) for w in block.w13], [np64(w) for w in block.w2]
    args = (np64(b["u"]), np64(b["layer"].logits), np64(b["h"]), np64(b["rstd"]), np64(dy), np64(torch.zeros_like(x) if dh is None else dh),
            np64(block.norm_weight), w_r, w13, w2)
    good = chain(*args)
    DX, DN, bwd, bound = good
    assert np.all(np.abs(np64(dx) - DX) <= bound), float(np.max(np.abs(np64(dx) - DX) / bound))
    assert max_rel(np64(g["norm"]), DN) <= BF16_BAR
    assert max_rel(np64(g["router"]), bwd["dw_r"]) <= BF16_BAR
    for k in range(len(WIDTHS)):
        assert max_rel(np64(g["w13"][k]), bwd["dw13"][k]) <= BF16_BAR
        assert max_rel(np64(g["w2"][k]), bwd["dw2"][k]) <= BF16_BAR
    if with_dh and T > 1:
        planted(good, args)


@pytest.mark.gpu
@pytest.mark.parametrize("part", ["both", "y", "h"])
def test_training_step_against_differences_along_the_gradient(part):
    """Along v = dx the derivative is |dx|^2: zero, a wrong sign or a missing part of the loss is off by as much as it is.
    The step (2^-4 of an element) leaves third-order terms of its square, 4e-3, and the BF16 outputs' rounding averages
    to below 1e-3 of the sum; 5e-2 covers both and the gradient's own 2e-2."""
    T = 256
    block, x, r, dy, dh = make(T, seed=9)
    dy = dy if part != "h" else torch.zeros_like(dy)
    dh = dh if part != "y" else torch.zeros_like(dh)
    block.train_forward(x, r)
    st = block._train
    idx = st.layer.expert_idx[:T].clone()
    B.layer_backward(block.cfg, st.layer, st.u, block.w_router, block.w13, block.w2, dy, aux=False)       # the loss has no aux term
    dx = torch.empty_like(x)
    B.mohge_norm_bwd(block.cfg, T, st.layer.dx, dh, st.h, block.norm_weight, st.rstd, dx, st.dnorm, False, st.layer.ws)
    step = 2.0 ** -4 * dx.float() / dx.float().square().mean(1, keepdim=True).sqrt()
    out = []
    for sign in (1, -1):
        xs = (x.float() + sign * step).bfloat16()
        y, h = block.train_forward(xs, r)
        out.append((xs.double(), y.double(), h.double(), (st.layer.expert_idx[:T] == idx).all(dim=1)))
    (xp, yp, hp, sp), (xm, ym, hm, sm) = out
    keep = (sp & sm)[:, None].double()               # tokens whose routing the step does not change
    assert keep.sum() >= T // 4
    want = float((((yp - ym) * dy.double() + (hp - hm) * dh.double()) * keep).sum())
    got = float((dx.double() * (xp - xm) * keep).sum())
    assert got > 0 and abs(want - got) <= 5e-2 * got, (want, got)
