"""The operators around the layer on buffers that begin on a 16-byte boundary and on no larger one: all that the header
asks of a pointer.  (The 8-bit experts store 32 bytes at a time where they may: that has to go by the buffer's address, not
by the row's length alone.)  Results are those on ordinary buffers, bit for bit."""
import pytest
import torch

import test_gpu_mx8 as mx8
import test_gpu_w4 as w4
from paper_2604_23108_b200 import binding as B

pytestmark = pytest.mark.gpu


def at16(t):
    """A copy of t whose address is 16 modulo 32."""
    n = 16 // t.element_size()
    raw = torch.empty(t.numel() + 2 * n, dtype=t.dtype, device="cuda")
    if raw.data_ptr() % 32 == 0:
        raw = raw[n:]
    out = raw[:t.numel()].view(t.shape)
    out.copy_(t)
    assert out.data_ptr() % 32 == 16
    return out


@pytest.mark.parametrize("cg", [1, 2])
@pytest.mark.parametrize("d,widths", [(256, [128, 256]), (264, [136, 24]), (1024, [352])])
def test_8_bit_experts(cg, d, widths):
    with mx8.forced_switches("MOHGE_TC_CG=%d" % cg):
        c = mx8.Case(200, d, widths, 2, 2, seed=d)
        plain = c.run().clone()
        b, w = c.b, c.w
        for name in ("xp8", "xp8_scale", "h8", "h8_scale", "y_perm", "y", "counts", "aligned", "tok_of_prow"):
            setattr(b, name, at16(getattr(b, name)))
        c.x8 = tuple(at16(t) for t in c.x8)
        w._set(*[[at16(t) for t in ts] for ts in (w.w13, w.w13_scale, w.w2, w.w2_scale)])
        assert torch.equal(c.run(), plain)


@pytest.mark.parametrize("T,d,gs", [(1, 264, 32), (9, 256, 64)])
def test_4_bit_experts(T, d, gs):
    c = w4.Case(T, d, [136, 24], 2, 2, gs)
    plain = c.run()
    c.x, c.idx, c.gate, c.scratch = (at16(t) for t in (c.x, c.idx, c.gate, c.scratch))
    q13, q2 = ([(at16(q), at16(s)) for q, s in x] for x in (c.q13, c.q2))
    c.w = B.W4Weights(c.cfg, gs, [a[0] for a in q13], [a[1] for a in q13], [a[0] for a in q2], [a[1] for a in q2])
    c.w.w13, c.w.w2 = [at16(t) for t in c.w.w13], [at16(t) for t in c.w.w2]
    c.w._a13, c.w._a2 = B._ptr_array(c.w.w13), B._ptr_array(c.w.w2)
    c.w.p13, c.w.p2 = B.C.cast(c.w._a13, B._P), B.C.cast(c.w._a2, B._P)
    y = at16(torch.zeros_like(c.x))
    B.mohge_expert_fwd_w4(c.cfg, T, c.x, c.idx, c.gate, c.w, c.scratch, y, c.ws)
    assert torch.equal(y, plain)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(3, 264), (40, 1024), (2, 4104)])
def test_norm(dtype, T, d):
    g = torch.Generator().manual_seed(d)
    n = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()  # noqa: E731
    cfg = B.Config(d, 1, 1, 1, 1, [8], dtype="bf16" if dtype == torch.bfloat16 else "f32", row_align=1)
    x, r, w, dy, dh = n(T, d), n(T, d), n(d), n(T, d), n(T, d)
    ws = B.new_workspace(cfg, T)
    got = []
    for f in (lambda t: t, at16):
        h, y, dx = (f(torch.zeros_like(x)) for _ in range(3))
        y8, s8 = (f(torch.zeros_like(t)) for t in B.mx8_empty(T, d))
        rstd, dw = f(torch.zeros(T, device="cuda")), f(torch.zeros(d, device="cuda"))
        B.mohge_norm_fwd(cfg, T, f(x), f(r), f(w), 1e-6, h, y, y8, s8, rstd)
        B.mohge_norm_bwd(cfg, T, f(dy), f(dh), h, f(w), rstd, dx, dw, False, f(ws))
        got.append((h, y, y8, s8, rstd, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*got))
