"""Latent attention's operators as a program calls them: one after the other in both forms, captured and replayed, on streams of their own,
over batches of many sequences."""
import math
import random

import pytest
import torch

from tests import latent_util as U

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2602_16603_amd import binding
    return binding


class Layer:
    """Projections of one layer in bf16 and what its operators are called with."""

    def __init__(self, heads, latent, rope, nope, v, max_position=600, seed=0):
        self.heads, self.latent, self.rope, self.nope, self.v = heads, latent, rope, nope, v
        self.w_ukv = U.normal((heads, nope + v, latent), seed + 1, latent ** -0.5)          # rows of the up projection, head by head
        self.gain = (1 + 0.1 * U.normal((latent,), seed + 2).float()).bfloat16()
        self.cos, self.sin = U.rope_tables(max_position, rope)
        self.max_position, self.scale = max_position, (nope + rope) ** -0.5
        self.dev = {k: getattr(self, k).cuda() for k in ("w_ukv", "gain", "cos", "sin")}
        self.dev["w_uk_t"] = self.w_ukv[:, :nope].transpose(1, 2).contiguous().cuda()      # laid out once

    def append(self, B, cache, pool, batch, x, q, q_out, at, stream=0):
        """q, q_out [T, H, *]: rotated parts from column nope of q to column `at` of q_out."""
        d = self.dev
        B.fp_op_latent_append(cache.struct(B, pool), batch, x.data_ptr(), x.stride(0), d["gain"].data_ptr(), 1e-6, x.shape[0], d["cos"].data_ptr(),
                              d["sin"].data_ptr(), self.max_position, B.FP_ROPE_INTERLEAVED, self.heads, q[..., self.nope:].data_ptr(), q.stride(0),
                              q.stride(1), q_out[..., at:].data_ptr(), q_out.stride(0), q_out.stride(1), stream)

    def absorbed(self, B, cache, pool, batch, x, q, max_new, max_len, ws, stream=0):
        """The cache with the new tokens, their outputs [T, H, V]; ws: (address, bytes)."""
        t, h, d = q.shape[0], self.heads, self.dev
        q_abs = torch.empty((t, h, self.latent + self.rope), dtype=torch.bfloat16, device="cuda")
        o_lat = torch.empty((t, h, self.latent), dtype=torch.bfloat16, device="cuda")
        o = torch.empty((t, h, self.v), dtype=torch.bfloat16, device="cuda")
        self.append(B, cache, pool, batch, x, q, q_abs, self.latent, stream)
        B.fp_op_gemm_heads(q.data_ptr(), q.stride(0), q.stride(1), d["w_uk_t"].data_ptr(), d["w_uk_t"].stride(0), q_abs.data_ptr(), q_abs.stride(0),
                           q_abs.stride(1), t, h, self.latent, self.nope, stream)
        B.fp_op_latent_attention(cache.struct(B, pool), batch, q_abs.data_ptr(), q_abs.stride(0), o_lat.data_ptr(), o_lat.stride(0), t, h, self.scale,
                                 max_new, max_len, ws[0], ws[1], stream)
        w_uv = d["w_ukv"][:, self.nope:]
        B.fp_op_gemm_heads(o_lat.data_ptr(), o_lat.stride(0), o_lat.stride(1), w_uv.data_ptr(), w_uv.stride(0), o.data_ptr(), o.stride(0), o.stride(1),
                           t, h, self.v, self.latent, stream)
        return o

    def expanded(self, B, cache, pool, batch, cu_q, lens, x, q, max_new, stream=0):
        t, h, rows, d = q.shape[0], self.heads, sum(lens), self.dev
        cu = torch.tensor([0] + list(lens)).cumsum(0).int().cuda()
        q_rot = q.clone()
        self.append(B, cache, pool, batch, x, q_rot, q_rot, self.nope, stream)
        lat = torch.empty((rows, self.latent), dtype=torch.bfloat16, device="cuda")
        kr = torch.empty((rows, self.rope), dtype=torch.bfloat16, device="cuda")
        B.fp_op_latent_gather(cache.struct(B, pool), batch, cu.data_ptr(), rows, lat.data_ptr(), kr.data_ptr(), stream)
        kv = torch.empty((rows, h, self.nope + self.v), dtype=torch.bfloat16, device="cuda")
        B.fp_op_gemm(1, lat.data_ptr(), d["w_ukv"].data_ptr(), kv.data_ptr(), rows, h * (self.nope + self.v), self.latent, 0, stream)
        o = torch.empty((t, h, self.v), dtype=torch.bfloat16, device="cuda")
        need = B.fp_op_latent_expanded_attention_workspace_bytes(t, len(lens), h, self.v, max_new, max(lens))
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        B.fp_op_latent_expanded_attention(cu_q.data_ptr(), cu.data_ptr(), len(lens), q_rot.data_ptr(), q_rot.stride(0), kv.data_ptr(), kv.stride(0),
                                          kr.data_ptr(), kr.stride(0), o.data_ptr(), o.stride(0), t, rows, h, self.nope, self.rope, self.v, self.scale,
                                          max_new, max(lens), ws.data_ptr() if need else 0, need, stream)
        torch.cuda.synchronize()
        return o

    def reference(self, x, q, positions):
        """x [L, R + P]: all tokens of a sequence before their norm; q [n, H, N + P] of the positions -> (o, tolerance), nothing rounded.

        With u half a bf16 step: a rounding of latents, rotated parts, absorbed queries or projected keys by u each moves a score by at most
        4 u times the sum of its products' sizes (three factors of a product are rounded, and fp32's own errors are far below a fourth),
        so a probability by a factor of exp(2 d) for the largest such d; probabilities are rounded (u, and u in their sum); values
        are off by 2 u of the projection's sizes (latent, value or sum), the output by u."""
        u, R, N = U.HALF_BF16, self.latent, self.nope
        c = x[:, :R].double()
        c = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6) * self.gain.double()
        kr, _ = U.rotate(x[:, R:].double(), self.cos[:len(x)], self.sin[:len(x)], True)
        w = self.w_ukv.double()
        out = torch.zeros((len(positions), self.heads, self.v), dtype=torch.float64)
        tol = torch.zeros_like(out)
        for i, p in enumerate(positions):
            qn = q[i, :, :N].double()
            qr, _ = U.rotate(q[i, :, N:].double(), self.cos[p], self.sin[p], True)
            k, v = (torch.einsum("lr,hnr->hln", c[:p + 1], m) for m in (w[:, :N], w[:, N:]))
            size_c, size_v = torch.einsum("hn,hnr->hr", qn.abs(), w[:, :N].abs()), torch.einsum("lr,hnr->hln", c[:p + 1].abs(), w[:, N:].abs())
            s = (torch.einsum("hn,hln->hl", qn, k) + qr @ kr[:p + 1].T) * self.scale
            d = 4 * u * self.scale * (size_c @ c[:p + 1].abs().T + qr.abs() @ kr[:p + 1].abs().T).amax(-1)
            pr = torch.softmax(s, -1)
            out[i] = torch.einsum("hl,hlv->hv", pr, v)
            rel = torch.expm1(2 * d) + 2 * u / (1 - u) + 4 * u
            tol[i] = u * out[i].abs() + rel[:, None] * torch.einsum("hl,hlv->hv", pr, size_v) * (1 + u)
        return out, tol


@pytest.mark.parametrize("heads,latent,rope,nope,v", [(4, 128, 32, 64, 64), (5, 512, 64, 128, 128), (70, 256, 32, 64, 128)])
def test_prompts_and_steps_in_both_forms(heads, latent, rope, nope, v):
    """Prompts, a second chunk and single tokens: append, products, absorbed attention, products; append, gather, projection,
    expanded attention.  Both against the definition, which knows neither form."""
    B = _binding()
    layer = Layer(heads, latent, rope, nope, v)
    total = [90, 33]
    cache = U.Cache(U.blocks_for(total, [0, 0]), latent, rope, garbage=math.nan)
    whole = U.Batch(total, [0, 0], cache.n, seed=heads)
    pools = [cache.pool.cuda(), cache.pool.cuda()]
    x, q = [U.normal((n, latent + rope), 10 + i, 2.0) for i, n in enumerate(total)], [U.normal((n, heads, nope + rope), 20 + i) for i, n in enumerate(total)]
    done = [0, 0]
    for new in ([40, 30], [48, 0], [1, 1], [1, 2]):
        b = U.Batch(new, done, cache.n)
        b.width, b.table = whole.width, whole.table
        st = b.struct(B)
        xs = torch.cat([x[s][done[s]:done[s] + n] for s, n in enumerate(new)]).cuda()
        qs = torch.cat([q[s][done[s]:done[s] + n] for s, n in enumerate(new)]).cuda()
        lens = [d + n for d, n in zip(done, new)]
        need = B.fp_op_latent_attention_workspace_bytes(sum(new), 2, heads, latent, rope, max(new), max(lens))
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        got = layer.absorbed(B, cache, pools[0], st, xs, qs, max(new), max(lens), (ws.data_ptr() if need else 0, need))
        torch.cuda.synchronize()
        other = layer.expanded(B, cache, pools[1], st, b.dev[0], lens, xs, qs, max(new))
        assert torch.equal(pools[0].nan_to_num(), pools[1].nan_to_num())
        lo = 0
        for s, n in enumerate(new):
            ref, tol = layer.reference(x[s], q[s][done[s]:done[s] + n], range(done[s], done[s] + n))
            U.check(got[lo:lo + n], ref, tol, ("absorbed", new, s))
            U.check(other[lo:lo + n], ref, tol, ("expanded", new, s))
            lo += n
        done = lens


@pytest.mark.parametrize("heads,max_new", [(20, 1), (70, 1), (4, 30)])
def test_captured_step_replays_on_new_lengths(heads, max_new):
    """One step captured once in two graphs with workspaces of their own; every replay has other lengths, tokens and idle slots, with eager
    work and synchronisation between, and gives the bits of the eager calls.  The two are replayed side by side too."""
    B = _binding()
    latent, rope, nope, v, seqs, width = 256, 32, 64, 64, 6, 64
    layer = Layer(heads, latent, rope, nope, v, width * 16)
    t = seqs * max_new
    cache = U.Cache(seqs * width, latent, rope, 4)
    table = torch.randperm(cache.n, device="cuda").int().view(seqs, width)
    cu = torch.arange(seqs + 1, device="cuda", dtype=torch.int32) * max_new
    cached = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    batch = B.fp_latent_batch(seqs, width, cu.data_ptr(), cached.data_ptr(), table.data_ptr())
    x = torch.zeros((t, latent + rope), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((t, heads, nope + rope), dtype=torch.bfloat16, device="cuda")
    need = B.fp_op_latent_attention_workspace_bytes(t, seqs, heads, latent, rope, max_new, width * 16)
    assert need > 0
    pools = [cache.pool.cuda() for _ in range(3)]
    ws = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs, graphs = [None] * 3, []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs[i] = layer.absorbed(B, cache, pools[i], batch, x, q, max_new, width * 16, (ws[i].data_ptr(), need),
                                     torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    side = torch.cuda.Stream()
    for r, lens in enumerate([[3, 700, -1, 15, 16, 40], [4, 701, 0, 500, 17, -1], [300, -1, -1, 2, 800, 33], [0] * 6, [-1, -1, -1, -1, -1, 600]]):
        cached.copy_(torch.tensor(lens, dtype=torch.int32))
        x.copy_(U.normal(tuple(x.shape), 200 + r))
        q.copy_(U.normal(tuple(q.shape), 300 + r))
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        outs[2] = layer.absorbed(B, cache, pools[2], batch, x, q, max_new, width * 16, (ws[2].data_ptr(), need), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[2]), r
        busy = torch.tensor(lens, device="cuda").repeat_interleave(max_new) >= 0
        for i in range(2):
            assert torch.equal(outs[i][busy], outs[2][busy]), r
        assert outs[2][busy].float().abs().sum() > 0


def test_calls_on_streams_of_their_own():
    """Two batches in both forms at once, each call on its own stream with its own workspace, give the bits they give alone."""
    B = _binding()
    cases = []
    for i, (new, cached, heads) in enumerate([([1] * 9, [100 * j + 600 for j in range(9)], 20), ([70, 90], [700, 20], 16)]):
        cache = U.Cache(U.blocks_for(new, cached), 256, 64, 50 + i)
        b = U.Batch(new, cached, cache.n, seed=i)
        q = U.normal((sum(new), heads, 320), 60 + i).cuda()
        need = B.fp_op_latent_attention_workspace_bytes(sum(new), len(new), heads, 256, 64, b.max_new, b.max_len)
        cases.append((cache, b, b.struct(B), cache.pool.cuda(), q, torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"), need))
    alone = [U.attend(B, c, pool, b, q, 0.05) for c, b, _, pool, q, _, _ in cases]
    structs = [c[1].struct(B) for c in cases]
    kv, kr, q2 = U.normal((900, 3, 256), 1).cuda(), U.normal((900, 64), 2).cuda(), U.normal((300, 3, 192), 3).cuda()
    alone.append(U.attend_expanded(B, [300], [900], q2, kv, kr, 128, 0.05))
    cu = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (300, 900)]
    need2 = B.fp_op_latent_expanded_attention_workspace_bytes(300, 1, 3, 128, 300, 900)
    ws2 = torch.empty(max(need2, 256), dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[torch.zeros_like(a) for a in alone] for _ in range(6)]
    torch.cuda.synchronize()
    for o in outs:
        for (c, b, _, pool, q, ws, need), st, out, stream in zip(cases, structs, o, streams):
            B.fp_op_latent_attention(c.struct(B, pool), st, q.data_ptr(), q.stride(0), out.data_ptr(), out.stride(0), q.shape[0], q.shape[1], 0.05,
                                     b.max_new, b.max_len, ws.data_ptr(), need, stream.cuda_stream)
        B.fp_op_latent_expanded_attention(cu[0].data_ptr(), cu[1].data_ptr(), 1, q2.data_ptr(), q2.stride(0), kv.data_ptr(), kv.stride(0), kr.data_ptr(),
                                          kr.stride(0), o[2].data_ptr(), o[2].stride(0), 300, 900, 3, 128, 64, 128, 0.05, 300, 900, ws2.data_ptr(), need2,
                                          streams[2].cuda_stream)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, alone))


@pytest.mark.parametrize("heads,most_new,most_cached", [(4, 1, 900), (20, 3, 300), (70, 2, 120)])
def test_many_ragged_sequences_that_share_blocks(heads, most_new, most_cached):
    """150 sequences of odd lengths, empty and idle ones among them; every third reads the first blocks of its neighbour."""
    B = _binding()
    rng = random.Random(heads)
    n = 150
    new = [rng.choice([0, 1, 1, 1, most_new]) for _ in range(n)]
    cached = [rng.choice([-1, 0, rng.randint(1, 40), rng.randint(0, most_cached)]) for _ in range(n)]
    latent, rope = 128, 32
    cache = U.Cache(U.blocks_for(new, cached), latent, rope, 7)
    batch = U.Batch(new, cached, cache.n, seed=3)
    for s in range(1, n, 3):
        for b in range(min(max(cached[s], 0) // 16, max(cached[s - 1], 0) // 16)):
            batch.table[s][b] = batch.table[s - 1][b]
    q = U.normal((sum(new), heads, latent + rope), 5)
    ref, tol = cache.attention(batch, q, 0.08)
    for workspace in (True, 0):
        got = U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), 0.08, workspace=workspace)
        U.check(got, ref, tol, workspace)


def test_a_long_cache_of_one_token():
    """65000 positions, cut into the most parts that a slot is cut into, with infinities of scores among them left out by their blocks."""
    B = _binding()
    latent, rope, heads, length = 128, 64, 3, 65000
    cache = U.Cache(U.blocks_for([1], [length]), latent, rope, 8)
    batch = U.Batch([1], [length], cache.n, seed=9)
    q = U.normal((1, heads, latent + rope), 6)
    for b in range(100, 3000, 7):
        cache.pool[batch.table[0][b]] = math.inf
        batch.table[0][b] = -1
    ref, tol = cache.attention(batch, q, 0.1)
    U.check(U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), 0.1), ref, tol)
