"""The operators of latent attention in 64 bits on the CPU, written from their definitions one token at a time, and the bounds of what
fp32 sums and roundings to bf16 may add."""
from __future__ import annotations

import math

import torch

from tests.kv8_util import BLOCK, HALF_BF16, HALF_FP32, Batch, blocks_for, check, rope_tables  # noqa: F401


def normal(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).bfloat16()


class Cache:
    """pool [N][16][R + P], bf16."""

    def __init__(self, blocks, latent, rope, seed=0, garbage=None):
        self.n, self.latent, self.rope = blocks, latent, rope
        self.pool = normal((blocks, BLOCK, latent + rope), seed) if garbage is None else torch.full((blocks, BLOCK, latent + rope), garbage).bfloat16()

    def struct(self, B, dev):
        return B.fp_latent_cache(dev.data_ptr(), self.n, self.latent, self.rope)

    def visible(self, batch, s):
        """Positions of sequence s whose block is there, and their rows in 64 bits."""
        n, c = batch.new[s], batch.cached[s]
        have = [b for b in range(min(batch.width, -(-(c + n) // BLOCK))) if 0 <= batch.table[s][b] < self.n] if c >= 0 else []
        if not have:
            return torch.zeros(0, dtype=torch.long), torch.zeros((0, self.latent + self.rope), dtype=torch.float64)
        key = torch.cat([torch.arange(b * BLOCK, b * BLOCK + BLOCK) for b in have])
        rows = torch.cat([self.pool[batch.table[s][b]] for b in have]).double()
        return key[key < c + n], rows[key < c + n]

    def attention(self, batch, q, scale, tokens=None):
        """-> (o [T, H, R], tolerance)."""
        tokens = q.shape[0] if tokens is None else tokens
        out = torch.zeros((*q.shape[:2], self.latent), dtype=torch.float64)
        tol = torch.zeros_like(out)
        for s in range(len(batch.new)):
            key, rows = self.visible(batch, s)
            for i in range(min(batch.cu[s + 1], tokens) - batch.cu[s]):
                sees = rows[key <= batch.cached[s] + i]
                out[batch.cu[s] + i], tol[batch.cu[s] + i] = softmax_sum(q[batch.cu[s] + i].double(), sees, sees[:, :self.latent], scale)
        return out, tol


def softmax_sum(q, k, v, scale):
    """q [H, D] over keys k [L, D] and values v [L, V] (or k [H, L, D], v [H, L, V]) -> (o, tolerance).

    Probabilities have a relative error u of half a bf16 step, and the sum that divides is taken over the rounded ones: o is off by at most
    2u/(1-u) sum p|v|.  The output's own rounding adds u |o|.  fp32 adds, as relative error of a probability, for its score (D + 4) half steps of
    sum |q k| scale, for the numerator and for the denominator; and a half step per key and a few for exp2 in the sums.  The matrix cores hold
    numbers below fp32's normal range as zero."""
    if k.shape[-2] == 0:
        zero = torch.zeros((q.shape[0], v.shape[-1]), dtype=torch.float64)
        return zero, zero.clone()
    per_head = k.dim() == 3
    w = torch.einsum("hd,hld->hl", q, k) if per_head else q @ k.T
    w = w * scale
    none = (w == -math.inf).all(-1, keepdim=True)
    p = torch.softmax(torch.where(none, 0.0, w), -1)
    o = torch.einsum("hl,hlv->hv", p, v) if per_head else p @ v
    o = torch.where(none, 0.0, o)
    kc, vc = k.abs().nan_to_num(posinf=0.0), v.abs().nan_to_num(posinf=0.0)
    size = (torch.einsum("hd,hld->hl", q.abs(), kc) if per_head else q.abs() @ kc.T) * scale
    spread = torch.einsum("hl,hlv->hv", p.nan_to_num(), vc) if per_head else p.nan_to_num() @ vc
    rel = 2 * HALF_BF16 / (1 - HALF_BF16) + 2 * (q.shape[-1] + 4) * HALF_FP32 * size.amax(-1, keepdim=True) + (k.shape[-2] + 16) * HALF_FP32
    return o, HALF_BF16 * o.abs().nan_to_num() + rel * spread * (1 + HALF_BF16) + 1e-35


def rotate(x, cos, sin, interleaved):
    """x [..., P] in 64 bits by angles [..., P/2]; -> (rotated, sum of the two products' sizes)."""
    half = x.shape[-1] // 2
    out, size = torch.zeros_like(x), torch.zeros_like(x)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = cos[..., j].double(), sin[..., j].double()
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def append(cache, batch, x, gain, eps, q, q_out, cos, sin, max_position, interleaved, tokens=None):
    """The definition on copies of the pool and q_out [T, H, P] -> (pool, tolerance, q_out, tolerance) in 64 bits; what is not written
    has no tolerance."""
    tokens = x.shape[0] if tokens is None else tokens
    pool, q_out = cache.pool.double(), q_out.double()
    pool_tol, q_tol = torch.zeros_like(pool), torch.zeros_like(q_out)
    R = cache.latent
    for s in range(len(batch.new)):
        for i in range(min(batch.cu[s + 1], tokens) - batch.cu[s]):
            t, pos = batch.cu[s] + i, batch.cached[s] + i
            if batch.cached[s] < 0 or pos >= max_position:
                continue
            q_out[t], size = rotate(q[t].double(), cos[pos], sin[pos], interleaved)
            q_tol[t] = HALF_BF16 * q_out[t].abs() + 4 * HALF_FP32 * size
            lb = pos // BLOCK
            blk = batch.table[s][lb] if lb < batch.width else -1
            if not 0 <= blk < cache.n:
                continue
            c = x[t, :R].double()
            tol = 0 * c
            if gain is not None:
                c = c / torch.sqrt((c * c).mean() + eps) * gain.double()
                # Sum of R squares (half its relative error in the root), the root, and three products.
                tol = (HALF_BF16 + (R / 2 + 8) * HALF_FP32) * c.abs()
            k, size = rotate(x[t, R:].double(), cos[pos], sin[pos], interleaved)
            pool[blk, pos % BLOCK] = torch.cat([c, k])
            pool_tol[blk, pos % BLOCK] = torch.cat([tol, HALF_BF16 * k.abs() + 4 * HALF_FP32 * size])
    return pool, pool_tol, q_out, q_tol


def expanded(new, lens, q, kv, k_rope, nope, scale, tokens=None, rows=None):
    """q [T, H, N + P], kv [L, H, N + V], k_rope [L, P] -> (o [T, H, V], tolerance)."""
    tokens = q.shape[0] if tokens is None else tokens
    rows = kv.shape[0] if rows is None else rows
    heads, v_dim = q.shape[1], kv.shape[2] - nope
    out = torch.zeros((q.shape[0], heads, v_dim), dtype=torch.float64)
    tol = torch.zeros_like(out)
    lo = at = 0
    for n, length in zip(new, lens):
        for i in range(min(n, tokens - lo)):
            end = min(max(length - n + i + 1, 0), max(rows - at, 0))
            x = kv[at:at + end].double().transpose(0, 1)
            k = torch.cat([x[..., :nope], k_rope[at:at + end].double().expand(heads, -1, -1)], -1)
            out[lo + i], tol[lo + i] = softmax_sum(q[lo + i].double(), k, x[..., nope:], scale)
        lo, at = lo + n, at + length
    return out, tol


# ---- on the GPU ----

def attend(B, cache, pool, batch, q, scale, workspace=True, o=None, tokens=None, max_new=None, max_len=None, stream=0, heads=None):
    """fp_op_latent_attention on device tensors q [T, H, R + P] and o [T, H, R] (token strides as they are); -> o."""
    tokens = q.shape[0] if tokens is None else tokens
    heads = q.shape[1]
    o = torch.full((q.shape[0], heads, cache.latent), 7.0, dtype=torch.bfloat16, device="cuda") if o is None else o
    max_new, max_len = max_new or batch.max_new, max_len or batch.max_len
    need = workspace
    if workspace is True:
        need = B.fp_op_latent_attention_workspace_bytes(tokens, len(batch.new), heads, cache.latent, cache.rope, max_new, max_len)
    ws = torch.full((max(need, 256) // 4,), math.nan, device="cuda")
    B.fp_op_latent_attention(cache.struct(B, pool), batch.struct(B), q.data_ptr(), q.stride(0), o.data_ptr(), o.stride(0), tokens, heads, scale,
                             max_new, max_len, ws.data_ptr() if need else 0, need, stream)
    torch.cuda.synchronize()
    return o


def attend_expanded(B, new, lens, q, kv, k_rope, nope, scale, workspace=True, o=None, tokens=None, rows=None, max_len=None, stream=0):
    tokens = q.shape[0] if tokens is None else tokens
    rows = kv.shape[0] if rows is None else rows
    heads, rope, v_dim = q.shape[1], q.shape[2] - nope, kv.shape[2] - nope
    o = torch.full((q.shape[0], heads, v_dim), 7.0, dtype=torch.bfloat16, device="cuda") if o is None else o
    cu = [torch.tensor([0] + list(v)).cumsum(0).int().cuda() for v in (new, lens)]
    max_new, max_len = max(list(new) + [1]), max_len or max(list(lens) + [1])
    need = workspace
    if workspace is True:
        need = B.fp_op_latent_expanded_attention_workspace_bytes(tokens, len(new), heads, v_dim, max_new, max_len)
    ws = torch.full((max(need, 256) // 4,), math.nan, device="cuda")
    B.fp_op_latent_expanded_attention(cu[0].data_ptr(), cu[1].data_ptr(), len(new), q.data_ptr(), q.stride(0), kv.data_ptr(), kv.stride(0),
                                      k_rope.data_ptr(), k_rope.stride(0), o.data_ptr(), o.stride(0), tokens, rows, heads, nope, rope, v_dim,
                                      scale, max_new, max_len, ws.data_ptr() if need else 0, need, stream)
    torch.cuda.synchronize()
    return o
