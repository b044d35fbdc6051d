"""One MoE layer in 8-bit integers or 4-bit floats, made of the library's calls.

    int8 weights                                        4-bit weights
    residual addition + RMS norm (bf16 and int8 rows)   (bf16 rows)           moe_rmsnorm
    experts and weights of each token                                         moe_route
    placement                                                                 moe_layout
                                                        4-bit rows            moe_quantize_mx
    int8 rows and their scales to the experts' windows  (4-bit rows)          moe_dispatch
    gate and up products, SwiGLU: moe_expert_matmul                           moe_expert_matmul_mx
    int8 rows of the result: moe_quantize               (4-bit rows)          moe_quantize_mx
    down product: moe_expert_matmul                                           moe_expert_matmul_mx
    weighted sum in token order                                               moe_combine

`MoeLayer` keeps the weights and the buffers of one batch shape; `forward`
enqueues the calls on a stream and allocates nothing, so that it can be
captured in a graph.  One GPU holds all experts (one rank).

python -m paper_2607_26444_amd.layer [--tokens N ...] [--mx] runs it on random inputs.
"""
from __future__ import annotations

import argparse
import contextlib
import sys

import torch

from . import moe

# scales of an int8 row, written once per block so that dispatch carries them
BLOCK = moe.MOE_FP8_BLOCK


class MoeLayer:
    """Weights of E experts and the buffers of a batch of T tokens.

    norm_weight [H] (bf16 or float32); w13 [E, 2I, H] int8, gate channels before
    up channels, w13_scale [E, 2I] float32; w2 [E, H, I] int8, w2_scale [E, H].
    Or 4-bit floats as moe_quantize_mx leaves them (H and I multiples of 32): w13
    [E, 2I, H/2] uint8, w13_scale [E, 2I, mx_scale_bytes(H)] uint8, w2 [E, H, I/2],
    w2_scale [E, H, mx_scale_bytes(I)]; the rows are then rounded to 4 bits as well.
    The routing's options are those of moe_route.
    """

    def __init__(self, T, H, I, E, k, norm_weight, w13, w13_scale, w2, w2_scale, bias=None,
                 eps=1e-6, score=moe.MOE_SCORE_SOFTMAX, groups=1, top_groups=1, group_top=1,
                 renorm=True, scale=1.0, device="cuda"):
        self.mx = w13.dtype == torch.uint8
        if self.mx:
            if H % moe.MOE_MX_BLOCK or I % moe.MOE_MX_BLOCK:
                raise ValueError(f"H and I have to be multiples of {moe.MOE_MX_BLOCK}")
            cols, inner_cols = moe.mx_scale_bytes(H), moe.mx_scale_bytes(I)
            weights = (("w13", w13, (E, 2 * I, H // 2), torch.uint8),
                       ("w13_scale", w13_scale, (E, 2 * I, cols), torch.uint8),
                       ("w2", w2, (E, H, I // 2), torch.uint8),
                       ("w2_scale", w2_scale, (E, H, inner_cols), torch.uint8))
        else:
            if H % BLOCK or I % 16:
                raise ValueError(f"H has to be a multiple of {BLOCK} and I of 16")
            weights = (("w13", w13, (E, 2 * I, H), torch.int8),
                       ("w13_scale", w13_scale, (E, 2 * I), torch.float32),
                       ("w2", w2, (E, H, I), torch.int8),
                       ("w2_scale", w2_scale, (E, H), torch.float32))
        for name, t, shape, dtype in (*weights,
                                      ("norm_weight", norm_weight, (H,), norm_weight.dtype),
                                      ("bias", bias, (E,), torch.float32)):
            if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or
                                  not t.is_contiguous()):
                raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {shape} is needed")
        self.T, self.H, self.I, self.E, self.k, self.eps = T, H, I, E, k, eps
        self.norm_weight, self.weight_dtype = norm_weight, _dtype(norm_weight)
        self.w13, self.w13_scale, self.w2, self.w2_scale = w13, w13_scale, w2, w2_scale
        self.bias = bias
        self.options = dict(score=score, groups=groups, top_groups=top_groups,
                            group_top=group_top, renorm=renorm, scale=scale)
        rows = max(1, T * k)

        def buf(*shape, dtype=torch.bfloat16):
            return torch.empty(*shape, dtype=dtype, device=device)
        self.sum, self.normed = buf(T, H), buf(T, H)
        if self.mx:
            # a row's scales behind its codes, so that dispatch carries both as one row; whole
            # lines of 128 bytes where they are an eighth more at most
            used, line = H // 2 + cols, -(-(H // 2 + cols) // 128) * 128
            self.row_bytes = line if 8 * line <= 9 * used else -(-used // 16) * 16
            self.q = buf(T, self.row_bytes, dtype=torch.uint8)
            self.rows = buf(rows, self.row_bytes, dtype=torch.uint8)
            self.q_scale, self.row_scale = self.q[:, H // 2:], self.rows[:, H // 2:]
            self.act_q = buf(rows, I // 2, dtype=torch.uint8)
            self.act_scale = buf(rows, inner_cols, dtype=torch.uint8)
        else:
            cols = H // BLOCK
            self.q, self.q_scale = buf(T, H, dtype=torch.int8), buf(T, cols, dtype=torch.float32)
            self.rows = buf(rows, H, dtype=torch.int8)
            self.row_scale = buf(rows, cols, dtype=torch.float32)
            self.act_q = buf(rows, I, dtype=torch.int8)
            self.act_scale = buf(rows, dtype=torch.float32)
        self.topk_idx = buf(T, k, dtype=torch.int32)
        self.topk_w = buf(T, k, dtype=torch.float32)
        self.layout = moe.Layout(T, k, E, 1, device=device)
        self.act = buf(rows, I)
        self.out = buf(rows, H)
        self.y = buf(T, H)
        # one rank: its regions are the tensors themselves
        tables = [t.data_ptr() for t in (self.rows, self.row_scale, self.out)]
        self.tables = torch.tensor(tables, dtype=torch.int64, device=device)
        self.row_table, self.scale_table, self.out_table = self.tables.split(1)
        self.cap = torch.tensor([rows], dtype=torch.int32, device=device)

    def forward(self, x, residual, logits, token_mask=None, stream=None):
        """x, residual [T,H] bf16 -> y [T,H] bf16, the layer's addition to the
        residual stream, which is left in `sum` (x + residual).  logits [T,E]
        float32 or bf16: a tensor, or a function of the normed rows [T,H] that
        makes it (the gate's product; its work goes to `stream` as well).
        token_mask [T] uint8: 0 for padding.  What is passed in has to be ready on
        `stream` and to stay until it has been read there."""
        T, H, I, E = self.T, self.H, self.I, self.E
        for name, t in (("x", x), ("residual", residual)):
            if tuple(t.shape) != (T, H) or t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ValueError(f"{name}: a contiguous bfloat16 tensor of shape {(T, H)} is needed")
        lay, rows = self.layout, T * self.k
        if self.mx:
            moe.moe_rmsnorm(x, residual, moe.MOE_DTYPE_BF16, self.norm_weight, self.weight_dtype,
                            self.eps, T, H, self.sum, self.normed, 0, None, None, None, 0, stream)
            moe.moe_quantize_mx(self.normed, T, H, self.q, self.q_scale, q_pitch=self.row_bytes,
                                scale_pitch=self.row_bytes, stream=stream)
        else:
            moe.moe_rmsnorm(x, residual, moe.MOE_DTYPE_BF16, self.norm_weight, self.weight_dtype,
                            self.eps, T, H, self.sum, self.normed if callable(logits) else None,
                            moe.MOE_DTYPE_INT8, self.q, self.q_scale, None, self.q_scale.shape[1],
                            stream)
        if callable(logits):
            with _current(stream):
                logits = logits(self.normed)
        # strides of single rows and columns say nothing; a pitch under E would be
        # rows that lie on each other (0, an expanded row, means packed to the call)
        pitch = logits.stride(0) if T > 1 and logits.dim() == 2 else E
        if tuple(logits.shape) != (T, E) or (E > 1 and logits.stride(1) != 1) or pitch < E:
            raise ValueError(f"logits: rows of {E} neighbouring values for {T} tokens are needed")
        if token_mask is not None and (tuple(token_mask.shape) != (T,) or
                                       token_mask.dtype != torch.uint8 or
                                       not token_mask.is_contiguous()):
            raise ValueError(f"token_mask: a contiguous uint8 tensor of {T} values is needed")
        moe.moe_route(logits, _dtype(logits), E, self.bias, token_mask, self.topk_idx,
                      self.topk_w, stream=stream, logits_pitch=pitch, **self.options)
        lay.run(self.topk_idx, stream)
        if self.mx:
            moe.moe_dispatch(self.q, None, moe.MOE_DTYPE_BF16, self.row_bytes // 2, E, 1,
                             self.topk_idx, lay.pos, lay.rank_offset, self.row_table, None, self.cap,
                             lay.workspace, lay.status, stream)
            moe.moe_expert_matmul_mx(self.rows, self.row_scale, rows, self.w13, self.w13_scale, E,
                                     2 * I, H, lay.expert_offset, lay.expert_count,
                                     moe.MOE_ACT_SWIGLU, self.act, stream, self.row_bytes,
                                     self.row_bytes)
            moe.moe_quantize_mx(self.act, rows, I, self.act_q, self.act_scale, row_src=lay.row_src,
                                stream=stream)
            moe.moe_expert_matmul_mx(self.act_q, self.act_scale, rows, self.w2, self.w2_scale, E, H,
                                     I, lay.expert_offset, lay.expert_count, moe.MOE_ACT_NONE,
                                     self.out, stream)
        else:
            moe.moe_dispatch(self.q, self.q_scale, moe.MOE_DTYPE_FP8_E4M3, H, E, 1, self.topk_idx,
                             lay.pos, lay.rank_offset, self.row_table, self.scale_table, self.cap,
                             lay.workspace, lay.status, stream)
            moe.moe_expert_matmul(self.rows, self.row_scale, rows, self.w13, self.w13_scale, E, 2 * I,
                                  H, lay.expert_offset, lay.expert_count, moe.MOE_ACT_SWIGLU, self.act,
                                  stream, self.row_scale.shape[1])
            moe.moe_quantize(self.act, rows, I, moe.MOE_DTYPE_INT8, self.act_q, self.act_scale,
                             lay.row_src, 1, stream)
            moe.moe_expert_matmul(self.act_q, self.act_scale, rows, self.w2, self.w2_scale, E, H, I,
                                  lay.expert_offset, lay.expert_count, moe.MOE_ACT_NONE, self.out,
                                  stream)
        moe.moe_combine(self.out_table, self.topk_w, H, E, 1, self.topk_idx, lay.pos,
                        lay.rank_offset, self.cap, self.y, lay.workspace, lay.status, stream)
        return self.y


def _current(stream):
    """Makes the stream that the calls are given torch's current one: what a
    function of the caller enqueues then lies between the calls, and what it
    allocates is not handed out again before the stream has read it."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    return torch.cuda.stream(stream)


def _dtype(t):
    if t.dtype == torch.float32:
        return moe.MOE_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return moe.MOE_DTYPE_BF16
    raise ValueError(f"bfloat16 or float32 is needed, not {t.dtype}")


def random_layer(T, H, I, E, k, seed=0, mx=False, **options):
    """A layer with weights of about unit gain; mx: in 4-bit floats."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def weights(n, depth):
        if mx:
            q = torch.empty(E, n, depth // 2, dtype=torch.uint8, device="cuda")
            scales = torch.empty(E, n, moe.mx_scale_bytes(depth), dtype=torch.uint8, device="cuda")
            for e in range(E):
                w = torch.randn(n, depth, generator=g, device="cuda") / depth ** 0.5
                moe.moe_quantize_mx(w.bfloat16(), n, depth, q[e], scales[e])
            return q, scales
        w = torch.randint(-127, 128, (E, n, depth), generator=g, device="cuda", dtype=torch.int8)
        return w, (0.5 + torch.rand(E, n, generator=g, device="cuda")) / (73.0 * depth ** 0.5)
    norm = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).bfloat16()
    return MoeLayer(T, H, I, E, k, norm, *weights(2 * I, H), *weights(H, I), **options)


def main(argv=None):
    ap = argparse.ArgumentParser(description="one MoE layer on random inputs")
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=7168)
    ap.add_argument("--inner", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--topk", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--mx", action="store_true", help="4-bit floats instead of 8-bit integers")
    a = ap.parse_args(argv)
    layer = random_layer(a.tokens, a.hidden, a.inner, a.experts, a.topk, mx=a.mx,
                         score=moe.MOE_SCORE_SIGMOID)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, residual = (torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16()
                   for _ in range(2))
    gate = torch.randn(a.hidden, a.experts, generator=g, device="cuda").bfloat16() / a.hidden ** 0.5

    def step():
        return layer.forward(x, residual, lambda normed: normed @ gate)
    step()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(a.steps):
        y = step()
    end.record()
    torch.cuda.synchronize()
    us = start.elapsed_time(end) * 1e3 / a.steps
    load = layer.layout.expert_count
    print(f"{a.tokens} tokens, {us:.1f} us a pass, rows per expert {int(load.min())} to "
          f"{int(load.max())}, mean square of y {float(y.float().square().mean()):.4f}, "
          f"status {int(layer.layout.status)}")


if __name__ == "__main__":
    sys.exit(main())
