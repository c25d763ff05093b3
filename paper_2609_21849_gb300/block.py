"""A transformer block around the quantized linears: norms with the residual's addition
and a quantized output, rotary positions on q and k, and linears with bias, activation
and residual in their epilogues, in FP8 (one scale per token) or NVFP4 (calibrated tensor
scales).

  a   = norm1(x)                          quantized
  qkv = a Wqkv^T + b                      q, k rotated in place
  o   = attention(q, k, v) Wout^T + b
  x1  = x + o;  c = norm2(x1)             one call, c quantized
  u   = gelu(c Wup^T + b)                 only its quantized form is written
  y   = u Wdown^T + b + x1

Attention itself is the caller's: ``project`` gives q, k and v, ``finish`` takes what
attention made of them.  ``forward`` runs both with the values in attention's place (the
re-quantized value columns feed the out-projection, as in the linear stack).

Host-side orchestration only: every step runs in libqlin's kernels, on buffers made once.

  python -m paper_2609_21849_gb300.block [--fmt fp8|nvfp4] [--tokens M]

builds a block of the denoiser's sizes with seeded random weights and times it.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass, field

import torch

from . import qlin, synthetic

EPS = 1e-6


@dataclass
class Block:
    fmt: str                      # "fp8" or "nvfp4"
    M: int
    hidden: int
    heads: int
    mlp: int
    plan: qlin.RopePlan
    norm1: torch.Tensor
    norm2: torch.Tensor
    W: dict = field(default_factory=dict)          # qkv, out, up, down
    bias: dict = field(default_factory=dict)
    scale: dict = field(default_factory=dict)      # static scales: v, u; NVFP4 also a, c
    q: dict = field(default_factory=dict)          # quantized a, v, o, c, u
    qkv: torch.Tensor | None = None
    o: torch.Tensor | None = None
    x1: torch.Tensor | None = None
    y: torch.Tensor | None = None
    workspace: torch.Tensor | None = None

    def _linear(self, A, name, **kw):
        call = qlin.qlin_linear_fp8 if self.fmt == "fp8" else qlin.qlin_linear_nvfp4
        return call(A, self.W[name], self.bias[name], **kw)

    def _norm(self, x, weight, name, residual=None, sum_out=None, stream=None):
        if self.fmt == "fp8":
            return qlin.qlin_rmsnorm_fp8(x, weight, residual, EPS, sum_out, out=self.q[name], stream=stream)
        return qlin.qlin_rmsnorm_nvfp4(x, self.scale[name], weight, residual, EPS, sum_out, out=self.q[name],
                                       stream=stream)

    def project(self, x: torch.Tensor, positions: torch.Tensor, stream=None):
        """(q, k, v), each a [M, heads, head_dim] view of the QKV output, q and k rotated."""
        self._norm(x, self.norm1, "a", stream=stream)
        # the value columns' quantized form serves finish() without an attention
        self._linear(self.q["a"], "qkv", y=self.qkv, next_scale=self.scale["v"], y_q=self.q["v"],
                     rq_col0=2 * self.hidden, stream=stream)
        H, D = self.heads, self.hidden // self.heads
        heads = self.qkv.view(self.M, 3 * H, D)
        qk = heads[:, :2 * H]
        qlin.qlin_rope(qk, positions, self.plan, qk, stream=stream)
        return heads[:, :H], heads[:, H:2 * H], heads[:, 2 * H:]

    def finish(self, x: torch.Tensor, attended: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """The rest of the block on x, the block's input, and attention's output
        [M, hidden] bf16 (None: the values that project() left stand in)."""
        o = self.q["v"] if attended is None else self.q["o"]
        if attended is not None:
            if self.fmt == "fp8":
                qlin.qlin_quantize_act_fp8(attended, None, o, self.workspace, stream)
            else:
                qlin.qlin_quantize_act_nvfp4(attended, None, o, self.workspace, stream)
        self._linear(o, "out", y=self.o, stream=stream)
        self._norm(self.o, self.norm2, "c", residual=x, sum_out=self.x1, stream=stream)
        self._linear(self.q["c"], "up", act=qlin.QLIN_ACT_GELU_TANH, next_scale=self.scale["u"], y_q=self.q["u"],
                     stream=stream)
        self._linear(self.q["u"], "down", residual=self.x1, y=self.y, stream=stream)
        return self.y

    def forward(self, x: torch.Tensor, positions: torch.Tensor, stream=None) -> torch.Tensor:
        self.project(x, positions, stream)
        return self.finish(x, None, stream)

    def calibrate(self, x: torch.Tensor):
        """Post-training calibration on the GPU: the dynamic tensor scales of the block's
        activations on x become the static ones."""
        def static(name, value):
            t = self.q[name]
            if self.fmt == "fp8":
                q = qlin.qlin_quantize_act_fp8(value, None, None, self.workspace)
                self.scale[name].copy_(q.scale)
                return t if t.per_channel else q
            q = qlin.qlin_quantize_act_nvfp4(value, None, t, self.workspace)
            self.scale[name].copy_(q.tensor_scale)
            return q

        def norm(src, weight, name, residual=None):
            n, s = qlin.qlin_rmsnorm(src, weight, residual, EPS)
            if self.fmt == "fp8":
                return self._norm(src, weight, name, residual, s)[0], s
            return static(name, n), s

        a, _ = norm(x, self.norm1, "a")
        self._linear(a, "qkv", y=self.qkv)
        v = static("v", self.qkv[:, 2 * self.hidden:].contiguous())
        o, _ = self._linear(v, "out")
        c, _ = norm(o, self.norm2, "c", x)
        u, _ = self._linear(c, "up", act=qlin.QLIN_ACT_GELU_TANH)
        static("u", u)
        torch.cuda.synchronize()


def build_block(fmt: str, M: int, hidden: int = synthetic.HIDDEN, heads: int = 24, mlp: int = synthetic.MLP,
                axes=None, layout: str = "interleaved", seed: int = 0, weights: dict | None = None,
                device="cuda") -> Block:
    """Quantize a block's weights (offline) and allocate the buffers of M tokens.
    ``weights``: bf16 tensors qkv, out, up, down, their biases ("qkv.bias", ...), norm1 and
    norm2; by default seeded random ones.  ``axes``: the rotary width of each position
    axis (default: one axis, the whole head)."""
    if fmt not in ("fp8", "nvfp4"):
        raise ValueError("fmt must be 'fp8' or 'nvfp4'")
    if hidden % heads != 0:
        raise ValueError("hidden must be a multiple of heads")
    shapes = {"qkv": (3 * hidden, hidden), "out": (hidden, hidden), "up": (mlp, hidden), "down": (hidden, mlp)}
    if weights is None:
        g = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device=device)  # noqa: E731
        weights = {n: (0.02 * rnd(*s)).bfloat16() for n, s in shapes.items()}
        weights |= {n + ".bias": (0.02 * rnd(s[0])).bfloat16() for n, s in shapes.items()}
        weights |= {n: (1 + 0.1 * rnd(hidden)).bfloat16() for n in ("norm1", "norm2")}
    b = Block(fmt, M, hidden, heads, mlp, qlin.rope_plan(axes or hidden // heads, layout=layout, device=device),
              weights["norm1"], weights["norm2"])
    b.workspace = qlin.alloc_workspace(device)
    code = qlin.QLIN_FMT_FP8 if fmt == "fp8" else qlin.QLIN_FMT_NVFP4
    for n in shapes:
        b.W[n] = qlin.qlin_quantize_weight(weights[n], code, workspace=b.workspace)
        b.bias[n] = weights[n + ".bias"]
    # (o has a scale of its own in every call, a and c one per row in FP8)
    for n, width in (("a", hidden), ("v", hidden), ("o", hidden), ("c", hidden), ("u", mlp)):
        b.q[n] = (qlin.alloc_fp8(M, width, n in "ac", device) if fmt == "fp8"
                  else qlin.alloc_nvfp4(M, width, device))
        if n != "o":
            b.scale[n] = torch.ones(1, dtype=torch.float32, device=device)
    empty = lambda w: torch.empty((M, w), dtype=torch.bfloat16, device=device)  # noqa: E731
    b.qkv, b.o, b.x1, b.y = empty(3 * hidden), empty(hidden), empty(hidden), empty(hidden)
    torch.cuda.synchronize()
    return b


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--fmt", choices=("fp8", "nvfp4"), default="nvfp4")
    ap.add_argument("--tokens", type=int, default=synthetic.M_TOKENS)
    a = ap.parse_args()
    b = build_block(a.fmt, a.tokens, axes=(16, 56, 56))
    x = torch.randn(a.tokens, b.hidden, device="cuda").bfloat16()
    positions = torch.randint(0, 64, (a.tokens, 3), device="cuda", dtype=torch.int32)
    b.calibrate(x)
    b.forward(x, positions)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(x, positions)
    for _ in range(3):
        graph.replay()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(20):
        graph.replay()
    e1.record()
    e1.synchronize()
    status = qlin.qlin_sync_status()
    if status != 0:
        raise SystemExit(f"device status {qlin.qlin_status_str(status)}")
    print(f"block {a.fmt}, {a.tokens} tokens: {e0.elapsed_time(e1) * 1e3 / 20:.1f} us, "
          f"finite {bool(torch.isfinite(b.y.float()).all())}")


if __name__ == "__main__":
    main()
