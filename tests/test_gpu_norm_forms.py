"""The norm's forward in both of its forms at every block width: one piece of eight columns per thread (batches that fit the
GPU at once, up to 8192 columns) and four (larger batches).  Bars as in test_gpu_norm.py; and rows must not depend on the
batch they come in beyond the order of a sum."""
import numpy as np
import pytest
import torch

from oracle import block_ops as Q
from test_gpu_norm import DT, EPS, F32, ROUND, cfg_of, fwd, normal, np64

pytestmark = pytest.mark.gpu

# 148 SMs x 2048 pieces: the larger batch of each pair takes four pieces per thread
PAIRS = [(136, 17000, 18000), (1024, 2300, 2400), (1032, 2300, 2400), (2056, 1100, 1200), (4096, 590, 600), (4104, 580, 600),
         (5000, 480, 490), (8192, 290, 300), (8200, 3, 300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,small,large", PAIRS)
def test_both_forms(dtype, d, small, large):
    x = (normal(1, large, d) * torch.exp(normal(2, large, 1))).to(DT[dtype]).cuda()
    r = normal(3, large, d).to(DT[dtype]).cuda()
    w = (1 + 0.1 * normal(4, d)).to(DT[dtype]).cuda()
    cfg = cfg_of(d, dtype)
    H, Y, R = Q.norm_fwd(np64(x), np64(r), np64(w), EPS)
    nb = -(-d // 32)
    for T in (small, large):
        h, y, rstd, y8, s8 = fwd(cfg, x[:T].contiguous(), r[:T].contiguous(), w, mx8=True)
        assert np.all(np.abs(np64(h) - H[:T]) <= (ROUND[dtype] + 2.0 ** -23) * np.abs(H[:T]))
        assert np.all(np.abs(np64(rstd) - R[:T]) <= F32 * R[:T])
        assert np.all(np.abs(np64(y) - Y[:T]) <= (ROUND[dtype] + F32) * np.abs(Y[:T]) + 1e-30)
        s = np64(s8[:, :nb])
        lo, hi = Q.mx8_bytes(Y[:T] * (1 - F32)), Q.mx8_bytes(Y[:T] * (1 + F32))
        assert np.all((s == lo) | (s == hi))
        want = Y[:T] / Q.mx8_scales(s, d)
        step = np.exp2(np.maximum(np.frexp(want)[1] - 1, -6) - 3.0)
        code = np64(y8[:, :d].contiguous().view(torch.float8_e4m3fn))
        assert np.all(np.abs(code - want) <= 0.5 * step + 2 * F32 * np.abs(want))
        assert not y8[:, d:].any() and not s8[:, nb:].any()
