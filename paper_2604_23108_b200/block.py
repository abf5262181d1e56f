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
        self.form = self._values = self._alive = None

    @staticmethod
    def _values_of(tensors):
        """Where the values lie, and how often torch has counted a write to them (inference tensors count none)."""
        try:
            return [(t.data_ptr(), t._version) for t in tensors]
        except RuntimeError:
            return [(t.data_ptr(), None if t.is_inference() else t._version) for t in tensors]

    def stale(self, tensors):
        return self._values != self._values_of(tensors)

    def made_from(self, tensors):
        self._values = self._values_of(tensors)
        self._alive = [t.detach() for t in tensors]          # their storage too: the same address is the same storage

    def forget(self):
        self._values = None


class TrainState:
    """What a train_forward of up to `cap` tokens leaves for its train_backward, and the gradients of the weights.
    Forward and backward may be enqueued on different streams: each waits for the state's last use."""

    def __init__(self, cfg: B.Config, T: int, device):
        n = lambda *s, dt=cfg.torch_dtype: torch.empty(*s, dtype=dt, device=device)  # noqa: E731
        self.cap = max(1, T)
        self.layer = B.LayerBuffers(cfg, self.cap, device)
        self.u, self.rstd = n(self.cap, cfg.d_model), n(self.cap, dt=torch.float32)
        self.dnorm = n(cfg.d_model, dt=torch.float32)
        self.T = self.grads_T = self.h = self.dx = None       # tokens of the latest forward and of the latest backward
        self._home, self._event = B._stream(), torch.cuda.Event()
        self.leave()

    def enter(self):
        if B._stream() != self._last and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().wait_event(self._event)

    def leave(self):
        self._last = B._stream()
        if torch.cuda.is_current_stream_capturing():
            return
        self._event.record()
        if self._last != self._home:             # the allocator is told of a stream that it does not know uses them
            for v in (*vars(self).values(), *vars(self.layer).values()):
                for t in v if isinstance(v, list) else [v]:
                    if isinstance(t, torch.Tensor):
                        t.record_stream(torch.cuda.current_stream())


class MoeBlock:
    """norm_weight [d], w_router [N_g + N_e, d], w13[g] [N, 2 W_g, d], w2[g] [N, d, W_g], all of the config's type on the
    device (prompt and tokens: BF16).  x and residual are [T, d] of that type, T any number of tokens.  The forward
    methods return (y, h): the block's output and the residual stream that the next block adds to.

    Results are tensors of their own, which no later call writes, unless a caller gives prompt or tokens the pair to
    write, out=(y, h), h possibly x or residual (allocating them is 3 of some 35 us of host time for a token).  h is
    also what train_backward reads: leave it as it is until then.  Working buffers are kept, one set for each way of running and stream, as large as the largest batch
    so far (release() frees them); inside a CUDA graph every call has buffers of its own, from the graph's memory.
    train_backward belongs to the latest train_forward; for several forwards in flight give each a state of its own,
    train_state(T), and hand it to both calls.

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
        self._sets = {}                      # (way of running, stream): its buffers
        self._train = self._train_captured = self._graded = None

    def _low_bit(self, kept, fits, make):
        """The form in `kept`, made anew if the weights are not those it was made from."""
        tensors = [*self.w13, *self.w2]
        if fits(kept.form) and not kept.stale(tensors):
            return kept.form
        if torch.cuda.is_current_stream_capturing():
            return make()                        # part of the graph: nothing ran that a later call could use
        if kept.form is not None:
            torch.cuda.synchronize(self.norm_weight.device)      # other streams may still be reading it
        if fits(kept.form):
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

    def release(self):
        """Frees the working buffers (calls that use them have to be complete, or enqueued on the current stream)."""
        self._sets.clear()
        self._train = self._train_captured = self._graded = None

    def _tokens_of(self, x, other=None, names=("x", "residual")):
        T, shape, want = x.shape[0], x.shape, self.cfg.torch_dtype
        if len(shape) != 2 or shape[1] != self.cfg.d_model or x.dtype is not want:
            raise B.MohgeError("%s is %s %s, expected %s [T, %d]" % (names[0], x.dtype, tuple(shape), want, self.cfg.d_model))
        if other is not None and (other.shape != shape or other.dtype is not want):
            raise B.MohgeError("%s is %s %s, expected %s %s" % (names[1], other.dtype, tuple(other.shape), want, tuple(shape)))
        return T

    # ---- serving

    def _serving(self, kind, T):
        """Buffers of a prompt or tokens call: the stream's set, grown if the batch is the largest so far."""
        capturing = torch.cuda.is_current_stream_capturing()
        key = (kind, B._stream())
        s = None if capturing else self._sets.get(key)
        if s is None or s["cap"] < T:
            s = None
            if not capturing:
                self._sets.pop(key, None)        # freed before the larger one is made
            cfg, dev, f32, i32 = self.cfg, self.norm_weight.device, torch.float32, torch.int32
            n = lambda *sh, dt=torch.bfloat16: torch.empty(*sh, dtype=dt, device=dev)  # noqa: E731
            s = {"cap": T, "T": None, "u": n(T, cfg.d_model),
                 "route": (n(T, cfg.n_logits, dt=f32), n(T, cfg.k_groups, dt=i32), n(T, cfg.k_experts, dt=i32),
                           n(T, cfg.k_experts, dt=f32), n(T, cfg.n_groups, dt=f32), n(T, cfg.n_experts, dt=f32))}
            if kind == "prompt":
                s["experts"], s["u8"] = B.Mx8Buffers(cfg, T, dev), B.mx8_empty(T, cfg.d_model, dev)
                s["ws"] = s["experts"].ws
            else:
                s["ws"], s["scratch"] = B.new_workspace(cfg, T, dev), B.w4_scratch(cfg, T, dev)
            if not capturing:
                self._sets[key] = s
        if s["T"] != T:
            if B.mohge_workspace_bytes(self.cfg, T) > s["ws"].numel():    # not always less for fewer tokens
                s["ws"] = B.new_workspace(self.cfg, T, s["ws"].device)
                if kind == "prompt":
                    s["experts"].ws = s["ws"]
            b = s["view"] = {"u": s["u"][:T], "route": tuple(t[:T] for t in s["route"]), "ws": s["ws"]}
            if kind == "prompt":
                b["experts"], b["u8"] = s["experts"], tuple(t[:T] for t in s["u8"])
            else:
                b["scratch"] = s["scratch"]
            s["T"] = T
        return s["view"]

    def _outputs(self, x, out):
        if out is None:
            return torch.empty_like(x), torch.empty_like(x)
        self._tokens_of(x, out[0], ("x", "y"))
        self._tokens_of(x, out[1], ("x", "h"))
        return out

    def _norm(self, T, x, residual, u, h, u8=(None, None), rstd=None):
        B.mohge_norm_fwd(self.cfg, T, x, residual, self.norm_weight, self.eps, h, u, u8[0], u8[1], rstd)

    def _route(self, b, T):
        logits, group_idx, expert_idx, gate, gs, esp = b["route"]
        B.mohge_route(self.cfg, T, b["u"], self.w_router, None, None, logits, group_idx, expert_idx, gate, gs, esp, b["ws"])
        return expert_idx, gate

    def prompt(self, x, residual=None, out=None):
        T = self._tokens_of(x, residual)
        y, h = self._outputs(x, out)
        if T > 0:
            weights = self.mx8_weights
            b = self._serving("prompt", T)
            self._norm(T, x, residual, b["u"], h, b["u8"])
            expert_idx, gate = self._route(b, T)
            B.layer_forward_mx8(self.cfg, b["experts"], *b["u8"], expert_idx, gate, weights, T=T, y=y)
        return y, h

    def tokens(self, x, residual=None, out=None):
        T = self._tokens_of(x, residual)
        y, h = self._outputs(x, out)
        if T > 0:
            weights = self.w4_weights
            b = self._serving("tokens", T)
            self._norm(T, x, residual, b["u"], h)
            expert_idx, gate = self._route(b, T)
            B.mohge_expert_fwd_w4(self.cfg, T, b["u"], expert_idx, gate, weights, b["scratch"], y, b["ws"])
        return y, h

    # ---- training

    def train_state(self, T):
        """A state for forwards of up to T tokens that other forwards leave alone."""
        return TrainState(self.cfg, T, self.norm_weight.device)

    def _own_state(self, T):
        """The block's state, for a forward of T tokens."""
        if torch.cuda.is_current_stream_capturing():
            self._train_captured = self.train_state(T)
            return self._train_captured
        st = self._train
        if st is not None and st.cap < T:
            st = self._train = self._graded = None                # freed before the larger one is made
        if st is None:
            st = self._train = self.train_state(T)
        return st

    def train_forward(self, x, residual=None, state=None):
        T = self._tokens_of(x, residual)
        st = state or self._own_state(T)
        if T > st.cap:
            raise B.MohgeError("train_forward of %d tokens with a state for %d" % (T, st.cap))
        st.enter()
        L = st.layer
        st.T = None
        L.y, st.h = self._outputs(x, None)
        if T > 0:
            if B.mohge_workspace_bytes(self.cfg, T) > L.ws.numel():       # not always less for fewer tokens
                L.ws = B.new_workspace(self.cfg, T, L.ws.device)
            self._norm(T, x, residual, st.u, st.h, rstd=st.rstd)
            B.layer_forward(self.cfg, L, st.u, self.w_router, self.w13, self.w2, T=T)
        st.T = T
        st.leave()
        return L.y, st.h

    def train_backward(self, dy, dh=None, state=None):
        """Gradient of x (and of the residual) of the latest train_forward (of the state's, where one is given); dh is
        the gradient that reaches h on the residual stream.  Weight gradients: grads()."""
        T = self._tokens_of(dy, dh, ("dy", "dh"))
        st = state or (self._train_captured if torch.cuda.is_current_stream_capturing() else self._train)
        if st is None or st.T != T:
            raise B.MohgeError("train_backward of %d tokens: the latest train_forward of this state had %s"
                               % (T, "none" if st is None or st.T is None else st.T))
        self.requantize()                        # what follows a gradient is an update
        st.enter()
        L, st.dx = st.layer, torch.empty_like(dy)
        if T == 0:
            for g in (st.dnorm, L.dw_router, *L.dw13, *L.dw2):
                g.zero_()
        else:
            B.layer_backward(self.cfg, L, st.u, self.w_router, self.w13, self.w2, dy, T=T)
            B.mohge_norm_bwd(self.cfg, T, L.dx, dh, st.h, self.norm_weight, st.rstd, st.dx, st.dnorm, False, L.ws)
        st.grads_T = T
        st.leave()
        if state is None:
            self._graded = st
        return st.dx

    def grads(self, T=None, state=None):
        """The weights' gradients that the latest train_backward (of T tokens) wrote; the next one overwrites them."""
        st = state or self._graded
        if st is None or st.grads_T is None or T not in (None, st.grads_T):
            raise B.MohgeError("grads: no train_backward%s" % ("" if T is None else " of %d tokens" % T))
        return {"norm": st.dnorm, "router": st.layer.dw_router, "w13": st.layer.dw13, "w2": st.layer.dw2}

    def _buffers(self, kind, T):
        """The working buffers of a way of running, as a call of T tokens on this stream finds them."""
        if kind != "train":
            return self._serving(kind, T)
        st = self._train if self._train is not None and self._train.cap >= T else self._own_state(T)
        if st.dx is None or st.dx.shape[0] != T:
            st.dx = torch.empty(T, self.cfg.d_model, dtype=self.cfg.torch_dtype, device=st.u.device)
        return {"layer": st.layer, "u": st.u[:T], "h": st.h, "rstd": st.rstd[:T], "dx": st.dx, "dnorm": st.dnorm, "ws": st.layer.ws}


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
