"""One residual block around a sparse V-MoE layer, trained through libvmoe.

    h     = norm(x)                                   before the layer
    x_out = x + row_scale gate post(layer(h)),  h_out = norm(x_out)
    loss  = the caller's on h_out and x_out, plus the gate's balance and z losses

`SparseBlock` owns the stream, the norms' and the gate's parameters and their
gradients beside the layer's `LayerBuffers`, all allocated once; `forward`,
`backward` and `update` enqueue their calls on the current stream and allocate
nothing; `update` also waits for the update before it, to learn whether that one
was skipped. `python -m paper_2608_16188_amd.block` trains one on a fixed target.
"""
from __future__ import annotations

import argparse
import contextlib
import math
import time

import torch

from . import vmoe_train as T
from . import workloads as W
from .layer import LayerBuffers

NORMS = {"none": T.VMOE_NORM_NONE, "rms": T.VMOE_NORM_RMS, "layer": T.VMOE_NORM_LAYER}


def _current(stream):
    """Context in which `stream` is the current one: None, a handle, or anything
    with .cuda_stream, as the calls take it."""
    if stream is None:
        return contextlib.nullcontext()
    handle = getattr(stream, "cuda_stream", stream)
    # an ExternalStream of handle 0 would be a new stream
    return torch.cuda.stream(torch.cuda.ExternalStream(handle) if handle
                             else torch.cuda.default_stream())


class SparseBlock:
    def __init__(self, cfg: W.LayerConfig, inputs: dict, *, norm: str = "layer",
                 post_norm: str = "none", gate_init: float = 0.1, row_scale: bool = False,
                 w_balance: float = 0.01, w_z: float = 0.001, state_bits: int = 32,
                 weight_decay: float = 0.05, max_norm: float = 1.0, device="cuda"):
        """norm: rms or layer, of the layer's input and of x_out; post_norm: none,
        rms or layer, of the layer's output. row_scale: whether tokens have a scale
        for the layer's output (drop-path; `self.row_scale`, ones at first).
        state_bits: 32, or 8 to keep AdamW's moments of tensors of 16384 elements or
        more in 8 bits. The tokens in `inputs` are the stream's first content."""
        for name, value, allowed in (("norm", norm, ("rms", "layer")),
                                     ("post_norm", post_norm, ("none", "rms", "layer")),
                                     ("state_bits", state_bits, (8, 32))):
            if value not in allowed:
                raise ValueError(f"{name}: one of {allowed} is wanted, got {value!r}")
        self.layer = L = LayerBuffers(cfg, inputs, device)
        self.w_balance, self.w_z, self.max_norm = w_balance, w_z, max_norm
        N, G, d, E = max(cfg.n_tokens, 1), cfg.n_groups, cfg.d_model, cfg.n_experts
        act, f32, dev = L.x.dtype, torch.float32, L.device
        dt = L.shape.dtype

        def shape(post):
            return T.make_norm_shape(cfg.n_tokens, d, dt, pre_norm=NORMS[norm],
                                     post_norm=NORMS[post])

        self.in_shape, self.out_shape = shape("none"), shape(post_norm)
        new = lambda dtype, *s: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.x = L.x.clone()  # the stream; the layer's x becomes its norm
        self.x_out, self.h_out = new(act, N, d), new(act, N, d)
        self.in_stats, self.out_stats, self.post_stats = (new(f32, N, 2) for _ in range(3))
        self.row_scale = torch.ones(N, device=dev) if row_scale else None
        # parameters and gradients by name
        self.params = dict(in_w=torch.ones(d, dtype=act, device=dev),
                           out_w=torch.ones(d, dtype=act, device=dev),
                           gate=torch.full((d,), gate_init, dtype=act, device=dev))
        if norm == "layer":
            self.params.update(in_b=torch.zeros(d, dtype=act, device=dev),
                               out_b=torch.zeros(d, dtype=act, device=dev))
        if post_norm != "none":
            self.params["post_w"] = torch.ones(d, dtype=act, device=dev)
        if post_norm == "layer":
            self.params["post_b"] = torch.zeros(d, dtype=act, device=dev)
        self.grads = {k: new(f32, d) for k in self.params}
        for k in ("w1", "b1", "w2", "b2"):
            self.params[k], self.grads[k] = getattr(L, k), getattr(L, "d" + k)
        if L.dw_router is not None:
            self.params["w_router"], self.grads["w_router"] = L.w_router, L.dw_router
        # activations' gradients
        self.dx, self.dx_mid = new(act, N, d), new(act, N, d)
        self.losses, self.demand = new(f32, G, 2), new(torch.int32, G, E)
        self.dlogits = new(f32, N, E)
        ws = lambda n: new(torch.uint8, max(n, 16))  # noqa: E731
        self.norm_ws = ws(max(T.vmoe_block_norm_bwd_workspace_bytes(s)
                              for s in (self.in_shape, self.out_shape)))
        self.loss_ws = ws(T.vmoe_load_balance_loss_workspace_bytes(L.shape))
        # optimizer
        self.states = {}
        for k, p in self.params.items():
            bits = 8 if state_bits == 8 and p.numel() >= 16384 else 32
            self.states[k] = T.adamw_state(p, bits)
        self.plan = T.AdamWPlan([
            T.AdamWTensor(param=p, grad=self.grads[k], **self.states[k],
                          weight_decay=weight_decay if k in ("w1", "w2", "w_router") else 0.0)
            for k, p in self.params.items()], dev)
        self.clip = new(f32, 2)
        self.clip_ws = ws(T.vmoe_grad_norm_workspace_bytes(self.plan))
        self._steps = 0  # but for the last update, until its clip is on the host
        self._clip_host = torch.empty(2, pin_memory=True)
        self._clip_there, self._clip_pending = torch.cuda.Event(), False

    @property
    def steps(self) -> int:
        """Steps taken: updates but for those whose gradient norm was not finite,
        which change nothing. Waits until the last one's norm is known."""
        if self._clip_pending:
            self._clip_there.synchronize()
            self._clip_pending = False
            self._steps += not math.isnan(self._clip_host[1])
        return self._steps

    @steps.setter
    def steps(self, taken: int):
        self._clip_pending, self._steps = False, taken

    def forward(self, stream=None):
        """From self.x to self.x_out and self.h_out."""
        L, p = self.layer, self.params
        T.vmoe_block_norm_fwd(self.in_shape, self.x, None, None, None, None, None, p["in_w"],
                              p.get("in_b"), None, L.x, None, self.in_stats, stream)
        L.forward(stream=stream)
        T.vmoe_block_norm_fwd(self.out_shape, self.x, L.y, p.get("post_w"), p.get("post_b"),
                              p["gate"], self.row_scale, p["out_w"], p.get("out_b"), self.x_out,
                              self.h_out, self.post_stats, self.out_stats, stream)

    def backward(self, dh_out, dx_out=None, stream=None):
        """From the loss's gradients at h_out (f32) and, along the stream, at
        x_out (the stream's type, or None for 0) to self.grads and self.dx."""
        L, p, g = self.layer, self.params, self.grads
        T.vmoe_block_norm_bwd(self.out_shape, dx_out, dh_out, self.x_out, L.y, p.get("post_w"),
                              p.get("post_b"), p["gate"], self.row_scale, p["out_w"],
                              self.post_stats, self.out_stats, self.dx_mid, L.dy, g.get("post_w"),
                              g.get("post_b"), g["gate"], g["out_w"], g.get("out_b"), self.norm_ws,
                              stream)
        T.vmoe_load_balance_loss(L.shape, L.logits, L.logit_bias, L.noise, L.probs, L.expert_idx,
                                 None, self.w_balance, self.w_z, self.losses, self.demand, None,
                                 self.dlogits, self.loss_ws, stream)
        L.backward(stream=stream, dlogits=self.dlogits)
        T.vmoe_block_norm_bwd(self.in_shape, self.dx_mid, L.dx, self.x, None, None, None, None,
                              None, p["in_w"], None, self.in_stats, self.dx, None, None, None,
                              None, g["in_w"], g.get("in_b"), self.norm_ws, stream)

    def update(self, lr: float, seed: int = 0, stream=None, **hyper):
        """One AdamW step on the gradients of the last backward, their norm held
        to max_norm; hyper: beta1, beta2, eps. A norm that is not finite changes
        nothing and is not counted. Not to be captured in a graph (RuntimeError):
        forward and backward are."""
        with _current(stream):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("update cannot be captured: a graph would repeat the step "
                                   "number, and with it the learning rate, the bias corrections "
                                   "and the random numbers of 8-bit states")
            step = self.steps + 1
            T.vmoe_grad_norm(self.plan, self.max_norm, self.clip, self.clip_ws)
            T.vmoe_adamw(self.plan, lr, step=step, seed=seed, clip=self.clip, **hyper)
            self._clip_host.copy_(self.clip, non_blocking=True)
            self._clip_there.record()
            self._clip_pending = True


def train(cfg, inputs, target, steps, lr, report=None, **options):
    """Fits h_out to `target` in the mean square; returns the block and the
    losses of every step."""
    block = SparseBlock(cfg, inputs, **options)
    losses = []
    for k in range(steps):
        block.forward()
        diff = block.h_out.float() - target
        losses.append(diff.square().mean())
        block.backward(diff * (2 / diff.numel()))
        # a cosine from lr to a tenth of it
        block.update(lr * (0.55 + 0.45 * math.cos(math.pi * k / steps)), seed=1)
        if report:
            report(k, losses[-1], block)
    return block, torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", choices=list(W.CONFIGS), default="vitb16_bf16")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    cfg = W.CONFIGS[a.workload]
    inputs = W.make_inputs(cfg)
    gen = torch.Generator(device="cuda").manual_seed(0)
    target = torch.randn(cfg.n_tokens, cfg.d_model, device="cuda", generator=gen)

    def report(k, loss, block):
        if k % 10 == 0 or k == a.steps - 1:
            print(f"step {k:4d}  loss {float(loss):.4f}  balance {float(block.losses[:, 0].mean()):.3f}"
                  f"  gradient norm {float(block.clip[0]):.3g}", flush=True)

    start = time.perf_counter()
    train(cfg, inputs, target, a.steps, a.lr, report, state_bits=a.state_bits, row_scale=False)
    torch.cuda.synchronize()
    print(f"{a.workload}: {a.steps} steps in {time.perf_counter() - start:.2f} s")


if __name__ == "__main__":
    main()
