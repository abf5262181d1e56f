"""The low-bit forms of a block's weights follow the weights: every kind of change between two calls is in the second."""
import pytest
import torch

from paper_2604_23108_b200 import binding as B
from paper_2604_23108_b200.block import MoeBlock
from test_gpu_block import make

pytestmark = pytest.mark.gpu


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def both(block, x):
    return [run(x)[0].clone() for run in (block.prompt, block.tokens)]


def fresh(block):
    return MoeBlock(block.cfg, block.norm_weight, block.w_router, list(block.w13), list(block.w2), block.eps, block.w4_group)


def assign(block):
    block.w13 = [w * 0.5 for w in block.w13]


def assign_one(block):
    block.w2[1] = block.w2[1] * 2


def write(block):
    block.w13[1].mul_(-0.5)


def write_a_view(block):
    block.w2[0][1, 3:].zero_()


def storage(block):
    block.w2[0].data = block.w2[0] * 3


def uncounted(block):
    block.w13[0].data.mul_(2)
    block.requantize()


def training_step(block):
    """The update goes past torch's counter, as a kernel's writes do."""
    block.train_forward(normal(8, 5, 256))
    block.train_backward(normal(9, 5, 256))
    for w, g in zip(block.w13, block.grads(5)["w13"]):
        w.data.add_(g.bfloat16(), alpha=-0.1)


@pytest.mark.parametrize("change", [assign, assign_one, write, write_a_view, storage, uncounted, training_step])
def test_prompt_and_tokens_answer_with_the_weights_as_they_are(change):
    block, _ = make()
    x = normal(1, 5, 256)
    before = both(block, x)
    assert all(torch.equal(a, b) for a, b in zip(before, both(block, x)))
    change(block)
    after, want = both(block, x), both(fresh(block), x)
    assert all(torch.equal(a, b) for a, b in zip(after, want))
    assert not any(torch.equal(a, b) for a, b in zip(after, before))


def test_another_group_of_the_4_bit_form():
    block, _ = make()
    x = normal(1, 5, 256)
    a = block.tokens(x)[0].clone()
    block.w4_group = 32
    b = block.tokens(x)[0].clone()
    assert not torch.equal(a, b) and torch.equal(b, fresh(block).tokens(x)[0])


def test_forms_are_made_once_while_nothing_changes():
    block, _ = make()
    x = normal(1, 5, 256)
    both(block, x)
    n = B.mohge_launch_count()
    both(block, x)
    steady = B.mohge_launch_count() - n
    n = B.mohge_launch_count()
    both(block, x)
    assert B.mohge_launch_count() - n == steady
    f, g = block.mx8_weights, block.w4_weights
    write(block)
    n = B.mohge_launch_count()
    both(block, x)
    assert B.mohge_launch_count() - n > steady
    assert block.mx8_weights is f and block.w4_weights is g              # in place: a graph holds the addresses


def test_weights_made_under_inference_mode():
    block, _ = make()
    with torch.inference_mode():
        block.w13 = [w * 0.5 for w in block.w13]
        block.w2 = [w * 0.5 for w in block.w2]
        x = normal(1, 5, 256)
        a = both(block, x)
        block.w13[0].mul_(2)
        block.requantize()
        b = both(block, x)
        assert all(torch.equal(u, v) for u, v in zip(b, both(fresh(block), x)))
        assert not any(torch.equal(u, v) for u, v in zip(a, b))


def test_first_use_on_one_stream_then_on_another():
    block, _ = make()
    x = normal(1, 5, 256)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for st in (s, t):
        st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = [block.mx8_weights, block.w4_weights]
    with torch.cuda.stream(t):
        b = [w.w13[0].clone() for w in a]                # what a second stream finds, without waiting for the first
    torch.cuda.synchronize()
    assert all(torch.equal(w.w13[0], v) for w, v in zip(a, b))


def test_a_graph_captured_with_forms_out_of_date_answers_with_the_weights_at_replay():
    block, _ = make()
    x = normal(1, 5, 256)
    both(block, x)
    write(block)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = block.prompt(x)[0], block.tokens(x)[0]
    for change in (lambda: None, lambda: write(block)):
        change()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, both(fresh(block), x)))
