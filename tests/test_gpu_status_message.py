"""The decoded status word names the kernel whose wait gave up (the words are written by the host here; no wait runs out)."""
import pytest
import torch

from paper_2604_23108_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("site,name", [(3, "grouped GEMM kernel"), (23, "8-bit experts"), (41, "4-bit experts"), (51, "norm's backward")])
def test_a_wait_that_gave_up(site, name):
    ws = B.new_workspace(B.Config(64, 1, 1, 1, 1, [8]), 1)
    ws[:4].view(torch.int32)[0] = (1 << 24) | site
    rc, word = B.mohge_get_device_status_rc(ws)
    message = B.lib().mohge_last_error().decode()
    assert rc == B.MOHGE_ERR_TIMEOUT and word == (1 << 24) | site
    assert "site %d" % site in message and name in message
