"""The block's buffers: results that later calls leave alone, memory that the largest batch bounds, streams, graphs, several
forwards in flight.  Everything is compared bit for bit with a block of its own for each call."""
import pytest
import torch

from paper_2604_23108_b200 import binding as B
from paper_2604_23108_b200.block import MoeBlock
from test_gpu_block import make

pytestmark = pytest.mark.gpu


def normal(seed, T, d=256):
    return torch.randn(T, d, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def fresh(block):
    return MoeBlock(block.cfg, block.norm_weight, block.w_router, block.w13, block.w2, block.eps, block.w4_group)


def runs(block):
    return {"prompt": block.prompt, "tokens": block.tokens, "train": block.train_forward}


def alone(block, kind, x, r=None):
    """A call's result from a block that makes no other call."""
    return [t.clone() for t in runs(fresh(block))[kind](x, r)]


def step(block, x, r, dy, dh, state=None):
    y, h = block.train_forward(x, r, state=state)
    dx = block.train_backward(dy, dh, state=state)
    return [y, h, dx] + grads(block, state)


def grads(block, state=None):
    g = block.grads(state=state)
    return [g["norm"].clone(), g["router"].clone()] + [t.clone() for t in g["w13"] + g["w2"]]


def same(a, b):
    return len(a) == len(b) and all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("kind", ["prompt", "tokens", "train"])
def test_a_later_call_leaves_results_alone(kind):
    block, _ = make()
    run = runs(block)[kind]
    xs = [(normal(i, 7), normal(10 + i, 7)) for i in range(3)]
    got = [run(x, r) for x, r in xs]
    for (x, r), g in zip(xs, got):
        assert same(g, alone(block, kind, x, r))


@pytest.mark.parametrize("kind", ["prompt", "tokens"])
def test_outputs_of_the_callers(kind):
    block, _ = make()
    x, r = normal(1, 7), normal(2, 7)
    y, h = alone(block, kind, x, r)
    out = torch.zeros_like(x), torch.zeros_like(x)
    got = runs(block)[kind](x, r, out=out)
    assert got[0] is out[0] and got[1] is out[1] and same(out, (y, h))
    got = runs(block)[kind](x, r, out=(out[0].zero_(), r))               # the residual stream in place
    assert got[1] is r and same(got, (y, h))
    for bad in (out[0][:6], out[0].float()):
        with pytest.raises(B.MohgeError, match="h is"):
            runs(block)[kind](x, out=(out[1], bad))


def test_a_later_step_leaves_results_alone():
    block, _ = make()
    a = [normal(i, 9) for i in range(4)]
    b = [normal(10 + i, 9) for i in range(4)]
    ya, ha = block.train_forward(*a[:2])
    dxa = block.train_backward(*a[2:])
    step(block, *b)
    assert same([ya, ha, dxa], step(fresh(block), *a)[:3])


@pytest.mark.parametrize("kind", ["prompt", "tokens", "train"])
def test_memory_is_bounded_by_the_largest_batch(kind):
    block, _ = make()
    run = runs(block)[kind]
    run(normal(0, 400))
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for T in (1, 399, 17, 128, 400, 3, 250, 64):
        x = normal(T, T)
        assert same(run(x), alone(block, kind, x))
        del x
        torch.cuda.synchronize()
        # y and h of the last forward may still be held for its backward
        assert torch.cuda.memory_allocated() <= held + 4 * 400 * 256 * 2
    block.release()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() < held


def test_a_workspace_that_is_larger_for_fewer_tokens():
    block, _ = make()
    T = next(t for t in range(64, 8192, 64) if B.mohge_workspace_bytes(block.cfg, t) > B.mohge_workspace_bytes(block.cfg, t + 64))
    step(block, *(normal(i, T + 64) for i in range(4)))
    a = [normal(10 + i, T) for i in range(4)]
    assert same(step(block, *a), step(fresh(block), *a))
    for kind in ("prompt", "tokens"):
        runs(block)[kind](normal(0, T + 64))
        assert same(runs(block)[kind](a[0]), alone(block, kind, a[0]))


@pytest.mark.parametrize("kind", ["prompt", "tokens"])
def test_two_streams_at_once(kind):
    block, _ = make()
    run = runs(block)[kind]
    xs = [normal(i, 300 if kind == "prompt" else 8) for i in range(2)]
    want = [alone(block, kind, x) for x in xs]
    run(xs[0])
    streams = [torch.cuda.Stream() for _ in xs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(20):
        for s, x, out in zip(streams, xs, got):
            with torch.cuda.stream(s):
                out.append(run(x))
    torch.cuda.synchronize()
    assert all(same(g, w) for out, w in zip(got, want) for g in out)


def test_several_forwards_in_flight():
    block, _ = make()
    a, b = ([normal(10 * k + i, T) for i in range(4)] for k, T in ((1, 30), (2, 45)))
    sa, sb = block.train_state(45), block.train_state(45)
    ya = block.train_forward(*a[:2], state=sa)
    yb = block.train_forward(*b[:2], state=sb)
    dxa = block.train_backward(*a[2:], state=sa)
    dxb = block.train_backward(*b[2:], state=sb)
    assert same([*ya, dxa] + grads(block, sa), step(fresh(block), *a))
    assert same([*yb, dxb] + grads(block, sb), step(fresh(block), *b))


def test_a_backward_without_its_forward_is_refused():
    block, _ = make()
    x = normal(1, 8)
    with pytest.raises(B.MohgeError, match="had none"):
        block.train_backward(x)
    with pytest.raises(B.MohgeError, match="no train_backward"):
        block.grads()
    block.train_forward(x)
    block.train_forward(x[:5].contiguous())
    with pytest.raises(B.MohgeError, match="had 5"):
        block.train_backward(x)                      # its activations are gone
    block.train_backward(x[:5].contiguous())
    block.train_backward(x[:5].contiguous())         # once more for another dy is fine
    with pytest.raises(B.MohgeError, match="of 8 tokens"):
        block.grads(8)
    with pytest.raises(B.MohgeError, match="state for 4"):
        block.train_forward(x, state=block.train_state(4))


def test_forward_and_backward_on_different_streams():
    block, _ = make()
    a = [normal(i, 200) for i in range(4)]
    want = step(fresh(block), *a)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for st in (s, t):
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        with torch.cuda.stream(s):
            y, h = block.train_forward(*a[:2])
        with torch.cuda.stream(t):
            dx = block.train_backward(*a[2:])
            g = grads(block)
    torch.cuda.synchronize()
    assert same([y, h, dx] + g, want)


@pytest.mark.parametrize("kind", ["prompt", "tokens"])
def test_a_graph_keeps_its_buffers_when_larger_batches_come(kind):
    block, _ = make()
    run = runs(block)[kind]
    x = normal(1, 5)
    run(x)
    s = torch.cuda.Stream()                          # captured on the stream that has warmed up
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        y = run(x)
    for T in (300, 700):
        with torch.cuda.stream(s):
            run(normal(T, T))
        torch.cuda.synchronize()
        junk = torch.full((1 << 22,), float("nan"), device="cuda")        # lands where freed buffers were
        x.copy_(normal(T + 1, 5))
        g.replay()
        torch.cuda.synchronize()
        assert same(y, alone(block, kind, x)) and bool(junk.isnan().all())


def test_a_training_step_in_a_graph():
    block, _ = make()
    a = [normal(i, 40) for i in range(4)]
    step(block, *a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, h = block.train_forward(*a[:2])
        dx = block.train_backward(*a[2:])
    for t in a:
        t.copy_(t.flip(0))
    g.replay()
    torch.cuda.synchronize()
    assert same([y, h, dx] + grads(block), step(fresh(block), *a))


def test_no_tokens():
    block, _ = make()
    x = normal(1, 0)
    for run in runs(block).values():
        y, h = run(x, x)
        assert y.shape == h.shape == (0, 256)
    assert block.train_backward(x, x).shape == (0, 256)
    assert not any(t.any() for t in grads(block))
    a = [normal(i, 6) for i in range(4)]
    assert same(step(block, *a), step(fresh(block), *a))
    block.train_forward(x)
    block.train_backward(x)
    assert not any(t.any() for t in grads(block))


def test_a_training_step_of_an_fp32_layer():
    """Buffers of the config's type.  FP32 against the same step in BF16 on values that BF16 holds exactly."""
    block, _ = make()
    c = block.cfg
    cfg = B.Config(c.d_model, c.n_groups, c.experts_per_group, c.k_groups, c.k_experts, list(c.group_width), dtype="f32", row_align=1)
    wide = MoeBlock(cfg, block.norm_weight.float(), block.w_router.float(), [w.float() for w in block.w13], [w.float() for w in block.w2])
    a = [normal(i, 50) for i in range(4)]
    low, high = step(block, *a), step(wide, *[t.float() for t in a])
    assert all(t.dtype == torch.float32 for t in high[:3])
    routed = (block._train.layer.expert_idx == wide._train.layer.expert_idx).all(dim=1)
    assert routed.float().mean() > 0.9                       # BF16's rounding of the norm's output moves few tokens
    for u, v in zip(low[:3], high[:3]):
        assert float((u.float() - v)[routed].norm() / v[routed].norm()) <= 2e-2
    with pytest.raises(B.MohgeError, match="BF16"):
        wide.tokens(a[0].float())
