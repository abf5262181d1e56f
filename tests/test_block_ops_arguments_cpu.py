"""What the binding of the operators around the layer checks before anything reaches the library (no GPU: a call that gets
past the check under test is turned down by a later one)."""
import pytest
import torch

from paper_2604_23108_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2604_23108_b200.build import build
    build()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8, torch.float8_e4m3fn])
def test_quantizing_refuses_types_it_would_read_as_another_one(dtype):
    """A float16 checkpoint read as float32 is twice its allocation."""
    w = torch.zeros(2, 16, 64).to(dtype)
    for call in (lambda: B.quantize_w4(w, 32), lambda: B.quantize_mx8(w)):
        with pytest.raises(B.MohgeError, match=str(dtype)):
            call()


def test_quantizing_refuses_outputs_that_are_too_small():
    w = torch.zeros(2, 16, 64)
    u8, bf = (lambda *s: torch.zeros(*s, dtype=torch.uint8)), (lambda *s: torch.zeros(*s, dtype=torch.bfloat16))
    for q, s, text in ((u8(2, 16, 31), bf(2, 16, 2), "q holds"), (u8(2, 16, 32), bf(2, 16, 1), "scale holds")):
        with pytest.raises(B.MohgeError, match=text):
            B.mohge_quantize_w4(w, 32, q, s)
    n = B.mohge_mx8_tiled_bytes(2, 16, 64)
    for q, s, text in ((u8(2, 16, 63), u8(n), "q holds"), (u8(2, 16, 64), u8(n - 1), "scale_tiled holds")):
        with pytest.raises(B.MohgeError, match=text):
            B.mohge_quantize_mx8(w, q, s)
