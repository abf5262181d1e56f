"""Dispatch on either side of the batch up to which one block does all of it, against the oracle's counting sort."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2604_23108_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 31, 33, 1023, 1024, 1025, 2049])
@pytest.mark.parametrize("Ng,N,Ke", [(1, 1, 1), (2, 5, 3), (4, 32, 8), (8, 32, 12)])
def test_dispatch_and_the_row_map(T, Ng, N, Ke):
    cfg = B.Config(8, Ng, N, Ng, Ke, [8] * Ng)
    Ne = Ng * N
    g = torch.Generator().manual_seed(T + Ke)
    idx = torch.rand(T, Ne, generator=g).argsort(1)[:, :Ke].int().contiguous()
    want = O.dispatch(idx.numpy(), Ne, 128)
    rows = B.mohge_perm_rows(cfg, T)
    f = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    counts, offsets, aligned, row, prow, src, tok = f(Ne), f(Ne + 4), f(Ne + 4), f(T, Ke), f(T, Ke), f(T * Ke), f(rows + 128)
    ws = B.new_workspace(cfg, T)
    B.mohge_dispatch_indices(cfg, T, idx.cuda(), counts, offsets, aligned, row, prow, src, tok, ws)
    for got, name in ((counts, "counts"), (offsets[:Ne + 1], "offsets"), (aligned[:Ne + 1], "aligned_offsets"), (row, "row_of"),
                      (prow, "prow_of"), (src, "src_of")):
        assert np.array_equal(got.cpu().numpy(), want[name]), name
    m = np.full(rows + 128, T)
    m[want["prow_of"]] = np.arange(T)[:, None]
    assert np.array_equal(tok.cpu().numpy(), m)
    assert B.mohge_get_device_status(ws) == 0
