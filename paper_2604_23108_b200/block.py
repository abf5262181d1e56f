"""The operators around the layer, together: a pre-norm block  h = x + residual,  y = experts(norm(h)).

    python -m paper_2604_23108_b200.block [--workload cfg2_bf16] [--prompt 2048] [--tokens 1 16 64] [--calls 50]

`MoeBlock` runs it three ways with the same weights:
  train_forward / train_backward   16-bit experts, gradients of everything (mohge_norm_fwd, the layer, mohge_norm_bwd)
  prompt                           mohge_norm_fwd writes 16 and 8 bits; routing in 16, experts in 8 (mohge_expert_fwd_mx8)
  tokens                           a few tokens: experts with 4-bit weights (mohge_expert_fwd_w4)
The command prints the time of each and how far the low-bit outputs are from the 16-bit ones.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from .inputs import WORKLOADS, make_device_inputs


class _LowBit:
    """The experts' weights in a low-bit form, and which values of the 16-bit weights it was made from."""

    def __init__(self):
        self.form = self._seen = None

    @staticmethod
    def _version(t):
        return None if t.is_inference() else t._version      # inference tensors count no writes

    def stale(self, tensors):
        # the aliases keep their storage alive: the same address is the same storage
        return self._seen is None or len(self._seen) != len(tensors) or any(
            a.data_ptr() != t.data_ptr() or v != self._version(t) for (a, v), t in zip(self._seen, tensors))

    def made_from(self, tensors):
        self._seen = [(t.detach(), self._version(t)) for t in tensors]

    def forget(self):
        self._seen = None


class MoeBlock:
    """norm_weight [d], w_router [N_g + N_e, d], w13[g] [N, 2 W_g, d], w2[g] [N, d, W_g], all BF16 on the device.
    Every method returns (y, h): the block's output and the residual stream that the next block adds to.

    The low-bit forms of w13 and w2 are made when they are first needed and made anew, in place, after the weights have
    changed: after a train_backward, whose step will change them, after a write that torch has counted, when another
    tensor took their place or w4_group changed.  A write that torch does not count (through .data or a raw pointer, into
    an inference tensor), made since the last train_backward and the last low-bit call, has to be followed by
    requantize().  A CUDA graph reads the forms that were there when it was captured; if they are out of date at that
    point, it makes its own at every replay."""

    def __init__(self, cfg: B.Config, norm_weight, w_router, w13, w2, norm_eps: float = 1e-6, w4_group: int = 128):
        self.cfg, self.eps, self.w4_group = cfg, norm_eps, w4_group
        self.norm_weight, self.w_router, self.w13, self.w2 = norm_weight, w_router, w13, w2
        self._mx8, self._w4 = _LowBit(), _LowBit()
        self._bufs = {}

    def _low_bit(self, kept, fits, make):
        """The form in `kept`, made anew if the weights are not those it was made from."""
        tensors = [*self.w13, *self.w2]
        if fits(kept.form) and not kept.stale(tensors):
            return kept.form
        if torch.cuda.is_current_stream_capturing():
            return make()                        # part of the graph: nothing ran that a later call could use
        if fits(kept.form):
            torch.cuda.synchronize(self.norm_weight.device)      # other streams may still be reading it
            kept.form.requantize(self.cfg, self.w13, self.w2)
        else:
            kept.form = make()
        torch.cuda.current_stream().synchronize()                # any stream may use it from here on
        kept.made_from(tensors)
        return kept.form

    @property
    def mx8_weights(self):
        return self._low_bit(self._mx8, lambda f: f is not None, lambda: B.Mx8Weights.quantize(self.cfg, self.w13, self.w2))

    @property
    def w4_weights(self):
        return self._low_bit(self._w4, lambda f: f is not None and f.group_size == self.w4_group,
                             lambda: B.W4Weights.quantize(self.cfg, self.w4_group, self.w13, self.w2))

    def requantize(self):
        """The weights have changed: the next low-bit call makes their low-bit forms anew."""
        self._mx8.forget()
        self._w4.forget()

    def _buffers(self, kind, T):
        """Device buffers of one way of running and one batch size, allocated once."""
        key = (kind, T)
        if key not in self._bufs:
            cfg, dev = self.cfg, self.norm_weight.device
            n = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=dev)  # noqa: E731
            b = {"h": n(T, cfg.d_model), "u": n(T, cfg.d_model), "rstd": n(T, dt=torch.float32)}
            if kind == "train":
                b["layer"] = B.LayerBuffers(cfg, T, dev)
                b["dx"], b["dnorm"] = n(T, cfg.d_model), n(cfg.d_model, dt=torch.float32)
                b["ws"] = b["layer"].ws
            else:
                f32, i32 = torch.float32, torch.int32
                b["route"] = (n(T, cfg.n_logits, dt=f32), n(T, cfg.k_groups, dt=i32), n(T, cfg.k_experts, dt=i32),
                              n(T, cfg.k_experts, dt=f32), n(T, cfg.n_groups, dt=f32), n(T, cfg.n_experts, dt=f32))
                if kind == "prompt":
                    b["experts"] = B.Mx8Buffers(cfg, T, dev)
                    b["ws"] = b["experts"].ws
                    b["u8"] = B.mx8_empty(T, cfg.d_model, dev)
                else:
                    b["ws"] = B.new_workspace(cfg, T, dev)
                    b["scratch"], b["y"] = B.w4_scratch(cfg, T, dev), n(T, cfg.d_model)
            self._bufs[key] = b
        return self._bufs[key]

    def _norm(self, b, T, x, residual, u8=(None, None)):
        B.mohge_norm_fwd(self.cfg, T, x, residual, self.norm_weight, self.eps, b["h"], b["u"], u8[0], u8[1], b["rstd"])

    def _route(self, b, T):
        logits, group_idx, expert_idx, gate, gs, esp = b["route"]
        B.mohge_route(self.cfg, T, b["u"], self.w_router, None, None, logits, group_idx, expert_idx, gate, gs, esp, b["ws"])
        return expert_idx, gate

    def train_forward(self, x, residual=None):
        T = x.shape[0]
        b = self._buffers("train", T)
        self._norm(b, T, x, residual)
        return B.layer_forward(self.cfg, b["layer"], b["u"], self.w_router, self.w13, self.w2), b["h"]

    def train_backward(self, dy, dh=None):
        """Gradient of x (and of the residual) after train_forward on the same batch size; dh is the gradient that
        reaches h on the residual stream.  Weight gradients: grads()."""
        T = dy.shape[0]
        b = self._buffers("train", T)
        self.requantize()                        # what follows a gradient is an update
        B.layer_backward(self.cfg, b["layer"], b["u"], self.w_router, self.w13, self.w2, dy)
        B.mohge_norm_bwd(self.cfg, T, b["layer"].dx, dh, b["h"], self.norm_weight, b["rstd"], b["dx"], b["dnorm"], False, b["ws"])
        return b["dx"]

    def grads(self, T):
        b = self._buffers("train", T)
        return {"norm": b["dnorm"], "router": b["layer"].dw_router, "w13": b["layer"].dw13, "w2": b["layer"].dw2}

    def prompt(self, x, residual=None):
        T = x.shape[0]
        b = self._buffers("prompt", T)
        self._norm(b, T, x, residual, b["u8"])
        expert_idx, gate = self._route(b, T)
        return B.layer_forward_mx8(self.cfg, b["experts"], *b["u8"], expert_idx, gate, self.mx8_weights), b["h"]

    def tokens(self, x, residual=None):
        T = x.shape[0]
        b = self._buffers("tokens", T)
        self._norm(b, T, x, residual)
        expert_idx, gate = self._route(b, T)
        B.mohge_expert_fwd_w4(self.cfg, T, b["u"], expert_idx, gate, self.w4_weights, b["scratch"], b["y"], b["ws"])
        return b["y"], b["h"]


def _time(fn, calls):
    for _ in range(3):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(calls):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / calls


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="cfg2_bf16", choices=[k for k, w in WORKLOADS.items() if w.dtype == "bf16"])
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 16, 64])
    ap.add_argument("--calls", type=int, default=50)
    args = ap.parse_args()
    wl = WORKLOADS[args.workload]
    torch.cuda.set_device(0)
    cfg = B.Config(wl.d_model, wl.n_groups, wl.experts_per_group, wl.k_groups, wl.k_experts, list(wl.group_width))
    inp = make_device_inputs(wl, torch.device("cuda", 0))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(wl.seed + 2000)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    block = MoeBlock(cfg, (1 + 0.1 * normal(wl.d_model)).bfloat16(), inp["w_router"], inp["w13"], inp["w2"])
    rel = lambda a, b: float((a.float() - b.float()).norm() / b.float().norm())  # noqa: E731
    T = min(args.prompt, wl.T)
    x, res = inp["x"][:T].contiguous(), normal(T, wl.d_model).bfloat16()
    ref = block.train_forward(x, res)[0].clone()
    dy = inp["dy"][:T].contiguous()

    def train():
        block.train_forward(x, res)
        block.train_backward(dy, dy)

    print("%s: training step of %d tokens %.3f ms" % (wl.name, T, _time(train, args.calls)))
    print("%s: forward of %d tokens in 16 bits %.3f ms" % (wl.name, T, _time(lambda: block.train_forward(x, res), args.calls)))
    y = block.prompt(x, res)[0]
    print("%s: forward of %d tokens in 8 bits %.3f ms, %.3f of the 16-bit output away"
          % (wl.name, T, _time(lambda: block.prompt(x, res), args.calls), rel(y, ref)))
    for t in args.tokens:
        a, r = x[:t].contiguous(), res[:t].contiguous()
        y = block.tokens(a, r)[0]
        print("%s: %d token(s) in 4 bits %.1f us, %.3f of the 16-bit output away"
              % (wl.name, t, 1e3 * _time(lambda: block.tokens(a, r), args.calls), rel(y, ref[:t])))


if __name__ == "__main__":
    main()
