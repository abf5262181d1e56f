"""The norm's backward at the ends of FP32's range: products of finite numbers that leave it on the way to a finite gradient.
Bars as in test_gpu_norm.py (FP32 outputs: 2^-18 of the magnitudes that enter)."""
import numpy as np
import pytest
import torch

from oracle import block_ops as Q
from paper_2604_23108_b200 import binding as B
from test_gpu_norm import DT, F32, ROUND, cfg_of, normal, np64

pytestmark = pytest.mark.gpu


def bwd(dtype, dy, dh, h, w, rstd):
    T, d = h.shape
    cfg = cfg_of(d, dtype)
    dx, dw = torch.empty_like(h), torch.empty(d, device="cuda")
    B.mohge_norm_bwd(cfg, T, dy, dh, h, w, rstd, dx, dw, False, B.new_workspace(cfg, T))
    return dx, dw


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [72, 1024, 5000])
@pytest.mark.parametrize("with_dh", [True, False])
def test_a_row_beyond_the_range_of_its_squares_leaves_the_others_and_dweight_alone(dtype, d, with_dh):
    """h dy of row 3 overflows; its rstd is zero, so it has dx = dh and no part in dweight."""
    T = 9
    x, dy, dh = (normal(i, T, d).to(DT[dtype]).cuda() for i in (1, 2, 3))
    x[3] = 3e38
    dy[3] = 5.0
    dh = dh if with_dh else None
    w = (1 + 0.1 * normal(4, d)).to(DT[dtype]).cuda()
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda")
    B.mohge_norm_fwd(cfg_of(d, dtype), T, x, None, w, 1e-6, h, y, None, None, rstd)
    assert rstd[3] == 0 and not y[3].any()
    dx, dw = bwd(dtype, dy, dh, h, w, rstd)
    assert torch.equal(dx[3], torch.zeros_like(dx[3]) if dh is None else dh[3])
    rest = [t for t in range(T) if t != 3]
    sub = lambda t: None if t is None else t[rest].clone()  # noqa: E731
    dx2, dw2 = bwd(dtype, sub(dy), sub(dh), sub(h), w, sub(rstd))
    assert torch.equal(dx[rest], dx2)
    sums = np.sum(np.abs(np64(sub(dy)) * np64(sub(h)) * np64(sub(rstd))[:, None]), axis=0)
    assert np.all(np.abs(np64(dw) - np64(dw2)) <= (T + 16) * 2.0 ** -24 * sums)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-25, 1e-20, 1e12, 1e18])
def test_rows_whose_rstd_squared_leaves_the_range(dtype, size):
    """rstd is the inverse of the rows' size, given as mohge_norm_fwd would have written it for norm_eps = 0."""
    T, d = 5, 264
    h = (normal(1, T, d) * size).to(DT[dtype]).cuda()
    dy, w = normal(2, T, d).to(DT[dtype]).cuda(), (1 + 0.1 * normal(4, d)).to(DT[dtype]).cuda()
    rstd = torch.from_numpy(1 / np.sqrt(np.mean(np64(h) ** 2, axis=1))).float().cuda()
    dx, dw = bwd(dtype, dy, None, h, w, rstd)
    DX, DW = Q.norm_bwd(np64(dy), None, np64(h), np64(w), np64(rstd))
    rs = np64(rstd)[:, None]
    g, xh = np64(dy) * np64(w), np64(h) * rs
    mag = rs * (np.abs(g) + np.abs(xh) * np.mean(np.abs(g * xh), axis=1, keepdims=True))
    assert np.all(np.abs(np64(dx) - DX) <= ROUND[dtype] * np.abs(DX) + F32 * mag)
    assert np.all(np.abs(np64(dw) - DW) <= (T + 16) * 2.0 ** -24 * np.sum(np.abs(np64(dy) * xh), axis=0))
