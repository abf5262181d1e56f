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


CFG = dict(d_model=64, n_groups=2, experts_per_group=3, k_groups=1, k_experts=2)


def weights(widths=(16, 32), N=3, d=64, dtype=torch.bfloat16, k=lambda n: n):
    z = lambda *s: torch.zeros(*s).to(dtype)  # noqa: E731
    return [z(N, 2 * w, k(d)) for w in widths], [z(N, d, k(w)) for w in widths]


@pytest.mark.parametrize("wrong,text", [
    (dict(widths=(16, 32, 8)), "3 w13 for 2 groups"), (dict(widths=(16,)), "1 w13 for 2 groups"),
    (dict(widths=(32, 16)), r"w13\[0\] is"), (dict(N=2), r"w13\[0\] is"), (dict(d=72), r"w13\[0\] is")])
def test_weights_of_another_layer_are_refused(wrong, text):
    """Surplus and missing groups, other widths, counts or columns: the library would read past their end."""
    cfg = B.Config(**CFG, group_width=[16, 32])
    w13, w2 = weights(**wrong)
    for make in (lambda: B.Mx8Weights.quantize(cfg, w13, w2), lambda: B.W4Weights.quantize(cfg, 32, w13, w2)):
        with pytest.raises(B.MohgeError, match=text):
            make()
    codes = weights(**wrong, dtype=torch.uint8)
    blocks = lambda n: -(-n // 32)  # noqa: E731
    with pytest.raises(B.MohgeError, match=text):
        B.Mx8Weights(cfg, codes[0], weights(**wrong, dtype=torch.uint8, k=blocks)[0], codes[1], weights(**wrong, dtype=torch.uint8, k=blocks)[1])
    q13, q2 = weights(**wrong, dtype=torch.uint8, k=lambda n: n // 2)
    s13, s2 = weights(**wrong, k=blocks)
    with pytest.raises(B.MohgeError, match=text):
        B.W4Weights(cfg, 32, q13, s13, q2, s2)


def test_codes_and_scales_of_another_form_are_refused():
    cfg = B.Config(**CFG, group_width=[16, 32])
    blocks = lambda n: -(-n // 32)  # noqa: E731
    c13, c2 = weights(dtype=torch.uint8)
    s13, s2 = weights(dtype=torch.uint8, k=blocks)
    with pytest.raises(B.MohgeError, match=r"codes: w13\[0\] is torch.bfloat16"):
        B.Mx8Weights(cfg, weights()[0], s13, c2, s2)
    with pytest.raises(B.MohgeError, match=r"scales: w2\[1\] is"):
        B.Mx8Weights(cfg, c13, s13, c2, [s2[0], s2[1][:, :32]])          # tiles would be read past their end
    with pytest.raises(B.MohgeError, match="scales are bytes"):
        B.mx8_tile_scales(torch.ones(1, 4, 2))
    one = B.mx8_tile_scales(torch.full((1, 4, 2), 130, dtype=torch.uint8).view(torch.float8_e8m0fnu))
    assert torch.equal(one, B.mx8_tile_scales(torch.full((1, 4, 2), 130)))
    q13, q2 = weights(dtype=torch.uint8, k=lambda n: n // 2)
    p13, p2 = weights(k=blocks)
    with pytest.raises(B.MohgeError, match=r"scales: w13\[0\] is torch.float32"):
        B.W4Weights(cfg, 32, q13, [s.float() for s in p13], q2, p2)
    with pytest.raises(B.MohgeError, match=r"codes: w2\[0\] is"):
        B.W4Weights(cfg, 32, q13, p13, [q[:, :, :4] for q in q2], p2)


def test_weights_are_refused_with_the_config_of_another_layer():
    cfg = B.Config(**CFG, group_width=[16, 32])
    w = B.Mx8Weights.__new__(B.Mx8Weights)
    w.layer = cfg.c().layer
    for other in (B.Config(**{**CFG, "n_groups": 3}, group_width=[16, 32, 8]), B.Config(**CFG, group_width=[16, 40])):
        with pytest.raises(B.MohgeError, match="weights of a layer"):
            B.mohge_expert_fwd_mx8(other, 1, None, None, None, None, w, None, None, None, None)
        with pytest.raises(B.MohgeError, match="weights of a layer"):
            B.mohge_expert_fwd_w4(other, 1, None, None, None, w, None, None, None)
    same = B.Config(**{**CFG, "k_experts": 1}, group_width=(16, 32))
    assert B._layer_of(same, w) is same.c()


def test_a_block_refuses_tokens_of_another_type_or_shape():
    from paper_2604_23108_b200.block import MoeBlock
    cfg = B.Config(**CFG, group_width=[16, 32])
    w13, w2 = weights()
    block = MoeBlock(cfg, torch.ones(64).bfloat16(), torch.zeros(8, 64).bfloat16(), w13, w2)
    x = torch.zeros(3, 64).bfloat16()
    for bad, args in (("x is torch.float32", (x.float(),)), ("x is torch.float16", (x.half(),)), (r"x is .*\(3, 56\)", (x[:, :56],)),
                      (r"residual is .*\(2, 64\)", (x, x[:2])), ("residual is torch.float32", (x, x.float()))):
        for call in (block.prompt, block.tokens, block.train_forward):
            with pytest.raises(B.MohgeError, match=bad):
                call(*args)
    with pytest.raises(B.MohgeError, match="dh is torch.float32"):
        block.train_backward(x, x.float())


def test_fewer_tokens_than_the_buffers_were_made_for():
    """The workspace is not always smaller for fewer tokens (the router backward's partial sums): checked, not assumed."""
    from types import SimpleNamespace
    cfg = B.Config(**{**CFG, "d_model": 1024}, group_width=[16, 32])
    T = next(t for t in range(64, 8192, 64) if B.mohge_workspace_bytes(cfg, t) > B.mohge_workspace_bytes(cfg, t + 64))
    b = SimpleNamespace(T=T + 64, ws=torch.empty(B.mohge_workspace_bytes(cfg, T + 64), dtype=torch.uint8))
    assert B._batch(cfg, b, None) == B._batch(cfg, b, T + 64) == T + 64 and B._batch(cfg, b, 1) == 1
    with pytest.raises(B.MohgeError, match="workspace"):
        B._batch(cfg, b, T)
    with pytest.raises(B.MohgeError, match="made for"):
        B._batch(cfg, b, T + 65)
