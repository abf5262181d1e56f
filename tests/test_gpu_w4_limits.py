"""4-bit experts at the widths the entry point accepts and at the sizes where its kernel changes form: two instead of four
tiles per copy (more tokens or columns than leave room for two such slots), rings of three, two and one slot, chunks of one,
two, four and eight tokens, a last tile that is not full.  Bars as in test_gpu_w4.py (sums over at most 8192 columns).

Forms, from what the tokens of a chunk leave of a block's shared memory:
  one or two tokens                       four tiles per copy at every width
  three to seven    groups of 32          two tiles per copy from some 6600 columns, 64: from some 8100
  eight and more    groups of 128, 64     two tiles per copy from some 4300 columns, 32: from some 3500
                    groups of 32, 8184+   a ring of one slot"""
import pytest
import torch

from test_gpu_w4 import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gs", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 2, 3, 9])
@pytest.mark.parametrize("d,widths", [
    (8192, [16, 40]),          # the first product's contraction at the limit, a second one of a single tile
    (8184, [136]),             # its last tile has 120 columns
    (16, [8192, 264]),         # the second product's contraction at the limit, beside a short one
    (24, [8184]),
    (4416, [4400]),            # both products where eight tokens begin to take two tiles per copy
    (6656, [24, 6616])])
def test_widths_up_to_the_limit(gs, T, d, widths):
    c = Case(T, d, widths, 2, 2, gs, seed=d + T)
    y = c.run()
    c.check(y)
    assert torch.equal(c.run(), y)


@pytest.mark.parametrize("gs", [32, 64, 128])
@pytest.mark.parametrize("d,widths", [(8192, [72]), (72, [8192])])
def test_a_full_pass_on_few_experts_at_the_limit(gs, d, widths):
    """64 tokens of three experts: every CTA begins several chunks of eight with the same, shortest ring."""
    c = Case(64, d, widths, 3, 2, gs, seed=gs)
    c.check(c.run())


def test_forms_side_by_side():
    """The same tokens in batches that run in different forms: nothing but the order of sums may differ."""
    c = Case(9, 8192, [40], 2, 2, 32, seed=5)
    y = c.run()
    for t in range(9):
        one = Case(1, 8192, [40], 2, 2, 32, seed=5, idx=c.idx[t:t + 1].cpu())
        one.x, one.gate, one.w = c.x[t:t + 1].clone(), c.gate[t:t + 1].clone(), c.w
        a, b = one.run().double(), y[t:t + 1].double()
        assert (a - b).abs().max() <= 2.0 ** -7 * b.abs().max()
