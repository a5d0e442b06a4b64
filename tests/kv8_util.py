"""The 8-bit KV cache in 64 bits on the CPU, written from its definition one block and one row at a time, and the same cache on the
GPU for the tests of its operators."""
from __future__ import annotations

import math

import torch

BLOCK, TOP = 16, 448.0
MIN_EXP, MAX_EXP = -110, 119
HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2
HALF_FP32 = torch.finfo(torch.float32).eps / 2


def e4m3(x):
    """Nearest e4m3 value: steps of 2^(e-3) in [2^e, 2^(e+1)), 2^-9 below 2^-6, ties to even, 448 at most, NaN stays."""
    mant, expo = torch.frexp(x)
    step = torch.tensor(2.0, dtype=torch.float64) ** (torch.clamp(expo, min=-5) - 4).double()
    y = torch.round(x / step) * step
    return torch.where(x.isnan(), x, torch.where(x.isinf(), torch.sign(x) * TOP, y.clamp(-TOP, TOP)))


def scale_of(amax: float) -> float:
    e = MIN_EXP
    while e < MAX_EXP and amax > TOP * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """k [N][Hkv][16][D] and v [N][Hkv][16][D] as codes in 64 bits (v not transposed), scales [N][Hkv]."""

    def __init__(self, blocks, hkv, dim, seed=0, garbage=None):
        g = torch.Generator().manual_seed(seed)
        self.n, self.hkv, self.dim = blocks, hkv, dim
        def codes():
            if garbage is not None:
                return torch.full((blocks, hkv, BLOCK, dim), garbage, dtype=torch.float64)
            return e4m3(torch.randn((blocks, hkv, BLOCK, dim), generator=g, dtype=torch.float64) * 60)
        def scales():
            return 2.0 ** torch.randint(-8, -4, (blocks, hkv), generator=g).double()
        self.code = {"k": codes(), "v": codes()}
        self.scale = {"k": scales(), "v": scales()}

    def value(self, name, blk, head):
        return self.code[name][blk, head] * self.scale[name][blk, head]

    def append(self, qkv, hq, cu, cached, table, cos, sin, max_position, q_out, tokens=None):
        hkv, dim, half = self.hkv, self.dim, self.dim // 2
        tokens = qkv.shape[0] if tokens is None else tokens
        x = qkv.double()
        for s in range(len(cached)):
            n = min(cu[s + 1], tokens) - cu[s]
            if cached[s] < 0 or n <= 0:
                continue
            n = min(n, max_position - cached[s])
            for lb in range(cached[s] // BLOCK, (cached[s] + n - 1) // BLOCK + 1 if n > 0 else 0):
                blk = table[s][lb] if lb < len(table[s]) else -1
                if not 0 <= blk < self.n:
                    continue
                lo, hi = max(lb * BLOCK, cached[s]), min(lb * BLOCK + BLOCK, cached[s] + n)
                rows = x[cu[s] + lo - cached[s]:cu[s] + hi - cached[s], :(hq + 2 * hkv) * dim].view(hi - lo, hq + 2 * hkv, dim)
                c, sn = cos[lo:hi].double()[:, None], sin[lo:hi].double()[:, None]
                a, b = rows[:, hq:hq + hkv, :half], rows[:, hq:hq + hkv, half:]
                new = {"k": torch.cat([a * c - b * sn, b * c + a * sn], -1), "v": rows[:, hq + hkv:]}
                for name, val in new.items():
                    for h in range(hkv):
                        w = val[:, h]
                        fin = w[w.isfinite()].abs()
                        sc = scale_of(fin.max().item() if fin.numel() else 0.0)
                        old = lo - lb * BLOCK
                        held = torch.zeros((BLOCK, dim), dtype=torch.float64)
                        if old:
                            before = self.scale[name][blk, h].item()
                            sc = max(sc, before)
                            held[:old] = e4m3(self.code[name][blk, h, :old] * (before / sc))
                        held[old:old + hi - lo] = e4m3(w / sc)
                        self.code[name][blk, h] = held
                        self.scale[name][blk, h] = sc
            for i in range(max(n, 0)):
                t, p = cu[s] + i, cached[s] + i
                r = x[t, :hq * dim].view(hq, dim)
                a, b, c, sn = r[:, :half], r[:, half:], cos[p].double(), sin[p].double()
                q_out[t, :hq * dim] = torch.cat([a * c - b * sn, b * c + a * sn], -1).reshape(-1)

    def attention(self, q, hq, cu, cached, table, scale, tokens=None):
        """-> (o [T, Hq*D], tolerance of every element).  With probabilities of relative error u = half a bf16 step and the sum
        taken over the rounded ones, o is off by at most 2u/(1-u) sum p|v|; the output's rounding adds u |o|; fp32 adds, as relative error
        of a probability, (D + 4) half steps of sum |q k| scale for its score (and twice that for numerator and denominator), and a half
        step per key and a few for exp2 in the sums."""
        tokens = q.shape[0] if tokens is None else tokens
        dim, group = self.dim, hq // self.hkv
        out = torch.zeros((q.shape[0], hq, dim), dtype=torch.float64)
        tol = torch.zeros_like(out)
        qd = q.double()[:, :hq * dim].reshape(q.shape[0], hq, dim)
        for s in range(len(cached)):
            n = min(cu[s + 1], tokens) - cu[s]
            if cached[s] < 0 or n <= 0:
                continue
            have = [b for b in range(min(len(table[s]), -(-(cached[s] + n) // BLOCK))) if 0 <= table[s][b] < self.n]
            if not have:
                continue
            key = torch.cat([torch.arange(b * BLOCK, b * BLOCK + BLOCK) for b in have])
            pos = cached[s] + torch.arange(n)
            sees = key[None, :] <= pos[:, None]
            for h in range(hq):
                k = torch.cat([self.value("k", table[s][b], h // group) for b in have])
                v = torch.cat([self.value("v", table[s][b], h // group) for b in have])
                rows = qd[cu[s]:cu[s] + n, h]
                w = torch.where(sees, rows @ torch.where(sees.any(0)[:, None], k, 0.0).T * scale, -math.inf)
                size = (rows.abs() @ k.abs().nan_to_num().T * scale).masked_fill(~sees, 0.0).amax(-1, keepdim=True)
                any_seen = sees.any(-1, keepdim=True)
                p = torch.where(any_seen, torch.softmax(w, -1), 0.0)
                nan = sees.double() @ v.isnan().double() > 0
                vz = v.nan_to_num()
                o = torch.where(any_seen, p @ vz, 0.0)
                spread = p @ vz.abs()
                rel = 2 * HALF_BF16 / (1 - HALF_BF16) + 2 * (dim + 4) * HALF_FP32 * size + (len(key) + 16) * HALF_FP32
                out[cu[s]:cu[s] + n, h] = torch.where(nan, math.nan, o)
                tol[cu[s]:cu[s] + n, h] = HALF_BF16 * o.abs() + rel * spread * (1 + HALF_BF16) + 1e-35
        return out.reshape(q.shape[0], -1), tol.reshape(q.shape[0], -1)

    # ---- on the GPU ----
    def upload(self):
        dev = {"k": self.code["k"].float().to(torch.float8_e4m3fn).cuda(),
               "v": self.code["v"].transpose(2, 3).contiguous().float().to(torch.float8_e4m3fn).cuda(),
               "ks": self.scale["k"].float().cuda(), "vs": self.scale["v"].float().cuda()}
        return dev

    def struct(self, B, dev):
        return B.fp_kv8_cache(dev["k"].data_ptr(), dev["v"].data_ptr(), dev["ks"].data_ptr(), dev["vs"].data_ptr(), self.n, self.hkv,
                              self.dim)

    def differs(self, dev):
        """Names of what the device copy does not hold bit for bit (NaN and the sign of zero apart)."""
        bad = []
        for name, got in (("k", dev["k"].float()), ("v", dev["v"].float().transpose(2, 3))):
            got = got.cpu().double()
            if not torch.equal(got.nan_to_num(nan=1e9), self.code[name].nan_to_num(nan=1e9)):
                bad.append(name)
            if not torch.equal(dev[name + "s"].cpu().double(), self.scale[name]):
                bad.append(name + "s")
        return bad


class Batch:
    """Lengths and block table of a packed batch, and their device copies; blocks are a permutation of the pool's."""

    def __init__(self, new, cached, blocks, seed=0, spare=0):
        g = torch.Generator().manual_seed(seed + 77)
        perm = torch.randperm(blocks, generator=g).tolist()
        self.new, self.cached = list(new), list(cached)
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        need = [-(-(max(c, 0) + n) // BLOCK) if c >= 0 else 0 for n, c in zip(new, cached)]
        self.width = max(need + [1]) + spare
        self.table, at = [], 0
        for nb in need:
            self.table.append(perm[at:at + nb] + [-1] * (self.width - nb))
            at += nb
        assert at <= blocks
        self.max_new = max(self.new)
        self.max_len = max([c + n for n, c in zip(new, cached) if c >= 0] + [1])

    def struct(self, B):
        self.dev = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (self.cu, self.cached, self.table)]
        return B.fp_kv8_batch(len(self.new), self.width, *(t.data_ptr() for t in self.dev))


def blocks_for(new, cached, spare=3):
    return sum(-(-(max(c, 0) + n) // BLOCK) for n, c in zip(new, cached)) + spare


def rope_tables(max_position, dim, theta=10000.0):
    angle = torch.arange(max_position, dtype=torch.float64)[:, None] * theta ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    return angle.cos().float(), angle.sin().float()


def attend(B, cache, dev, batch, q, hq, scale, workspace=True, o=None, tokens=None, max_new=None, max_len=None, stream=0):
    """fp_op_kv8_attention on device tensors q and o (row strides as they are); -> o."""
    tokens = q.shape[0] if tokens is None else tokens
    o = torch.full((q.shape[0], hq * cache.dim), 7.0, dtype=torch.bfloat16, device="cuda") if o is None else o
    max_new, max_len = max_new or batch.max_new, max_len or batch.max_len
    need = B.fp_op_kv8_attention_workspace_bytes(tokens, len(batch.new), hq, cache.hkv, cache.dim, max_new, max_len) if workspace is True else workspace
    ws = torch.full((max(need, 256) // 4,), math.nan, device="cuda")
    B.fp_op_kv8_attention(cache.struct(B, dev), batch.struct(B), q.data_ptr(), q.stride(0), o.data_ptr(), o.stride(0), tokens, hq, scale,
                          max_new, max_len, ws.data_ptr() if need else 0, need, stream)
    torch.cuda.synchronize()
    return o


def check(got, ref, tol, what=""):
    got = got.float().cpu().double()
    assert torch.equal(got.isnan(), ref.isnan()), what
    off = ((got - ref).abs() - tol).nan_to_num(nan=-1.0)
    assert (off <= 0).all(), (what, off.max().item(), (off > 0).sum().item())
