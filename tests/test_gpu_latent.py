"""The operators of latent attention, through the C ABI, against their definitions in 64 bits within bounds derived from the roundings that
are made (latent_util.py)."""
import math

import pytest
import torch

from tests import latent_util as U

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2602_16603_amd import binding
    return binding


BATCHES = [
    ([1], [0]), ([1], [15]), ([1], [31]), ([1], [32]), ([1, 1, 1], [63, 64, 1]), ([33], [0]), ([2, 0, 5, 1], [100, 20, 30, 0]),
    ([70], [45]), ([1] * 70, [5 * i for i in range(70)]),
]


# ---- append ----

@pytest.mark.parametrize("latent,rope,heads", [(512, 64, 20), (512, 32, 1), (256, 32, 40), (256, 64, 33), (128, 32, 4), (128, 64, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new,cached", BATCHES + [([5, 0, 33, 1], [3, 20, 14, -1])])
def test_append_matches_the_definition(latent, rope, heads, interleaved, new, cached):
    _append(latent, rope, heads, interleaved, new, cached, gain=True)


@pytest.mark.parametrize("gain", [True, False])
@pytest.mark.parametrize("in_place", [True, False])
def test_append_with_strides_missing_blocks_and_rows_behind_the_batch(gain, in_place):
    """A block outside the pool, a token beyond the table, one beyond the rotation tables, tokens that the call does not have."""
    _append(256, 32, 3, True, [20, 40, 6], [30, 7, 0], gain, in_place, pad=24, missing=[(0, 2), (1, 1)], cut=1, tokens=65, max_position=45)


def _append(latent, rope, heads, interleaved, new, cached, gain, in_place=False, pad=0, missing=(), cut=0, tokens=None, max_position=None):
    B = _binding()
    cache = U.Cache(U.blocks_for(new, cached), latent, rope, garbage=math.nan)
    batch = U.Batch(new, cached, cache.n, seed=latent + heads)
    for i, (s, b) in enumerate(missing):
        batch.table[s][b] = cache.n + 5 if i else -7
    if cut:
        batch.width -= cut
        batch.table = [row[:batch.width] for row in batch.table]
    t = sum(new)
    cos, sin = U.rope_tables(batch.max_len + 1, rope)
    max_position = max_position or batch.max_len + 1
    x, g = U.normal((t, latent + rope), 1, 3.0), U.normal((latent,), 2)
    q = U.normal((t, max(heads, 1), rope + pad), 3)
    q_out = q if in_place else torch.full_like(q, 5.0)
    pool, pool_tol, ref_q, q_tol = U.append(cache, batch, x, g if gain else None, 1e-6, q[..., :rope], q_out[..., :rope], cos, sin, max_position,
                                            interleaved, tokens)
    dev, xd, gd, qd, cd, sd = cache.pool.cuda(), torch.zeros((t, latent + rope + pad), dtype=torch.bfloat16, device="cuda"), g.cuda(), q.cuda(), cos.cuda(), sin.cuda()
    xd[:, :latent + rope] = x.cuda()
    od = qd if in_place else q_out.cuda()
    B.fp_op_latent_append(cache.struct(B, dev), batch.struct(B), xd.data_ptr(), xd.stride(0), gd.data_ptr() if gain else None, 1e-6,
                          t if tokens is None else tokens, cd.data_ptr(), sd.data_ptr(), max_position,
                          B.FP_ROPE_INTERLEAVED if interleaved else B.FP_ROPE_HALF, heads, qd.data_ptr(), qd.stride(0), qd.stride(1),
                          od.data_ptr(), od.stride(0), od.stride(1))
    torch.cuda.synchronize()
    U.check(dev, pool, pool_tol, "pool")
    if heads:
        U.check(od[..., :rope], ref_q, q_tol, "queries")
        assert torch.equal(od[..., rope:].cpu(), q_out[..., rope:])


@pytest.mark.parametrize("what", ["zeros", "tiny", "large", "nan", "inf"])
def test_append_extreme_rows(what):
    """A row of zeros is stored as zeros, one whose squares vanish in fp32 by eps alone; NaN and infinity stay in their own row."""
    B = _binding()
    cache = U.Cache(4, 256, 32)
    batch = U.Batch([3], [14], cache.n)
    cos, sin = U.rope_tables(32, 32)
    x, g = U.normal((3, 288), 4), U.normal((256,), 5)
    x[1] = {"zeros": 0.0, "tiny": 1e-30, "large": 1e17, "nan": 1.0, "inf": 1.0}[what]
    if what in ("nan", "inf"):
        x[1, 7] = math.nan if what == "nan" else math.inf
    pool, tol, _, _ = U.append(cache, batch, x, g, 1e-6, torch.zeros((3, 1, 32)), torch.zeros((3, 1, 32)), cos, sin, 32, False)
    dev, xd, gd, cd, sd = cache.pool.cuda(), x.cuda(), g.cuda(), cos.cuda(), sin.cuda()
    B.fp_op_latent_append(cache.struct(B, dev), batch.struct(B), xd.data_ptr(), 288, gd.data_ptr(), 1e-6, 3, cd.data_ptr(), sd.data_ptr(), 32,
                          B.FP_ROPE_HALF)
    torch.cuda.synchronize()
    U.check(dev, pool, tol + 1e-38)


# ---- gather ----

@pytest.mark.parametrize("latent,rope", [(512, 64), (512, 32), (256, 64), (128, 32)])
@pytest.mark.parametrize("lens", [[1], [8], [9], [16], [17, 0, 31], [100, 1, 48], [3] * 70])
def test_gather_is_exact(latent, rope, lens):
    B = _binding()
    cache = U.Cache(U.blocks_for(lens, [0] * len(lens)), latent, rope)
    batch = U.Batch(lens, [0] * len(lens), cache.n, spare=1)
    if len(lens) > 1 and lens[-1] > 16:
        batch.table[-1][1] = -1                        # positions of a block that is not there are zero
    total = sum(lens)
    out = [torch.full((total + 3, w), 9.0, dtype=torch.bfloat16, device="cuda") for w in (latent, rope)]
    dev, cu = cache.pool.cuda(), torch.tensor(batch.cu, dtype=torch.int32, device="cuda")
    B.fp_op_latent_gather(cache.struct(B, dev), batch.struct(B), cu.data_ptr(), total + 3, out[0].data_ptr(), out[1].data_ptr())
    torch.cuda.synchronize()
    ref = torch.full((total + 3, latent + rope), 9.0).bfloat16()
    for s, n in enumerate(lens):
        for i in range(n):
            blk = batch.table[s][i // 16]
            ref[batch.cu[s] + i] = cache.pool[blk, i % 16] if blk >= 0 else 0.0
    assert torch.equal(out[0].cpu(), ref[:, :latent]) and torch.equal(out[1].cpu(), ref[:, latent:])


def test_gather_of_fewer_rows_and_a_short_table():
    """Positions beyond the table are zero; rows from n_rows on are left as they were."""
    B = _binding()
    cache = U.Cache(3, 128, 64)
    batch = U.Batch([40], [0], cache.n)
    batch.width, batch.table = 2, [batch.table[0][:2]]
    out = [torch.full((40, w), 9.0, dtype=torch.bfloat16, device="cuda") for w in (128, 64)]
    dev, cu = cache.pool.cuda(), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    B.fp_op_latent_gather(cache.struct(B, dev), batch.struct(B), cu.data_ptr(), 37, out[0].data_ptr(), out[1].data_ptr())
    torch.cuda.synchronize()
    ref = torch.cat([cache.pool[batch.table[0][0]], cache.pool[batch.table[0][1]], torch.zeros((5, 192)), torch.full((3, 192), 9.0)]).bfloat16()
    assert torch.equal(torch.cat([o.cpu() for o in out], 1), ref)


# ---- absorbed attention ----

def _attention(latent, rope, heads, new, cached, seed=0, std=1.0, scale=None, evict=None, cache_of=None, edit=None, **kw):
    B = _binding()
    cache = U.Cache(U.blocks_for(new, cached), latent, rope, seed) if cache_of is None else cache_of
    batch = U.Batch(new, cached, cache.n, seed=seed)
    if evict:
        evict(batch, cache)
    # Slots of the pool that no position of the batch has hold NaN.
    used = torch.zeros((cache.n, 16), dtype=torch.bool)
    for s, (n, c) in enumerate(zip(new, cached)):
        for p in range(max(c, 0) + n if c >= 0 else 0):
            if p // 16 < batch.width and 0 <= batch.table[s][p // 16] < cache.n:
                used[batch.table[s][p // 16], p % 16] = True
    cache.pool[~used] = math.nan
    if edit:
        edit(cache, batch)
    q = U.normal((sum(new), heads, latent + rope), seed + 1, std)
    scale = scale or (latent + rope) ** -0.5
    ref, tol = cache.attention(batch, q, scale)
    got = U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), scale, **kw)
    U.check(got, ref, tol)
    return got


SHAPES = [(512, 64, 20), (512, 64, 16), (512, 32, 3), (256, 32, 40), (256, 64, 65), (128, 32, 4), (128, 64, 130), (512, 64, 128)]


@pytest.mark.parametrize("latent,rope,heads", SHAPES)
@pytest.mark.parametrize("new,cached", BATCHES)
def test_attention_matches_the_definition(latent, rope, heads, new, cached):
    _attention(latent, rope, heads, new, cached)


@pytest.mark.parametrize("latent,rope,heads", [(512, 64, 20), (512, 64, 128), (256, 32, 40), (128, 32, 4)])
@pytest.mark.parametrize("new,cached", [([1], [3000]), ([1, 1, 1], [2000, 17, 900]), ([3, 0, 4], [1500, 8, 700]), ([40], [1200]),
                                        ([1] * 66, [20 * i for i in range(66)])])
@pytest.mark.parametrize("workspace", [True, False, "some"])
def test_attention_of_keys_cut_into_shares(latent, rope, heads, new, cached, workspace):
    B = _binding()
    need = B.fp_op_latent_attention_workspace_bytes(sum(new), len(new), heads, latent, rope, max(new), max(c + n for c, n in zip(cached, new)))
    assert need > 0
    _attention(latent, rope, heads, new, cached, workspace=True if workspace is True else need // 5 // 256 * 256 if workspace else 0)


def _evict(batch, cache):
    for s, row in enumerate(batch.table):
        for b in range(1, len(row)):
            if (b + s) % 3 == 0:
                row[b] = [-1, cache.n, -2 ** 31, 2 ** 31 - 1][b % 4]


@pytest.mark.parametrize("latent,rope,heads", [(512, 64, 20), (256, 32, 40), (128, 64, 70)])
@pytest.mark.parametrize("new,cached", [([1, 1, 1, 1], [-1, 200, 5, -3]), ([40, 3, 1], [100, -1, 600]), ([1] * 5, [-1] * 5), ([2], [900])])
def test_attention_idle_sequences_and_missing_blocks(latent, rope, heads, new, cached):
    _attention(latent, rope, heads, new, cached, evict=_evict)


def test_attention_of_sequences_whose_blocks_are_all_gone():
    def gone(batch, cache):
        batch.table = [[-1] * batch.width for _ in batch.table]
    got = _attention(512, 64, 20, [1, 17], [400, 31], evict=gone)
    assert (got == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("latent,rope,heads", [(512, 64, 20), (128, 32, 4), (256, 64, 65)])
@pytest.mark.parametrize("new,cached", [([33], [0]), ([5, 40], [40, 3]), ([1, 1], [31, 600])])
def test_attention_what_is_not_finite_reaches_only_rows_that_see_it(latent, rope, heads, new, cached, bad):
    """Latents of the newest tokens, of one in the middle and, alone, a rotated part."""
    def edit(cache, batch):
        for s, (n, c) in enumerate(zip(new, cached)):
            for p, at in ((c + n - 1, 3), (c + n // 2, latent - 1), (c + n - 2, latent + 1)):
                if p >= 0:
                    cache.pool[batch.table[s][p // 16], p % 16, at] = bad
    _attention(latent, rope, heads, new, cached, edit=edit)


def test_attention_strides_padding_and_wrong_hints():
    """Longer rows, more rows than the batch has, hints that are too small and too large: the same rows, the others as they were."""
    B = _binding()
    new, cached, latent, rope, heads = [3, 20, 1], [40, 0, 700], 256, 32, 5
    cache = U.Cache(U.blocks_for(new, cached), latent, rope)
    batch = U.Batch(new, cached, cache.n)
    t = sum(new)
    q = U.normal((t + 6, heads, latent + rope), 1)
    ref, tol = cache.attention(batch, q, 0.05, t)
    wide = torch.full((t + 6, heads * (latent + rope) + 40), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :heads * (latent + rope)] = q.reshape(t + 6, -1).cuda()
    qd = wide[:, :heads * (latent + rope)].view(t + 6, heads, latent + rope)
    for max_new, max_len in ((20, 701), (1, 1), (300, 9000), (1, 9000)):
        buf = torch.full((t + 6, heads * latent + 16), 7.0, dtype=torch.bfloat16, device="cuda")
        o = buf[:, :heads * latent].view(t + 6, heads, latent)
        U.attend(B, cache, cache.pool.cuda(), batch, qd, 0.05, o=o, tokens=t + 6, max_new=max_new, max_len=max_len)
        U.check(o[:t], ref[:t], tol[:t], (max_new, max_len))
        assert (buf[t:] == 7).all() and (buf[:, heads * latent:] == 7).all()


def test_attention_of_positions_beyond_the_table_sees_all_of_it():
    B = _binding()
    cache = U.Cache(4, 256, 64)
    batch = U.Batch([2], [62], cache.n)
    q = U.normal((2, 8, 320), 3)
    ref = U.Batch([2], [62], cache.n)
    key, rows = cache.visible(ref, 0)
    want = [U.softmax_sum(q[i].double(), rows, rows[:, :256], 0.05) for i in range(2)]
    for cached in (64, 1000, 2 ** 31 - 5):
        batch.cached = [cached]
        got = U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), 0.05, max_new=2, max_len=64)
        U.check(got, torch.stack([w[0] for w in want]), torch.stack([w[1] for w in want]), cached)


@pytest.mark.parametrize("std,scale", [(300.0, 1.0), (1e6, 3.0), (1e-20, 1.0), (1.0, 1e30), (1.0, 1e-30)])
@pytest.mark.parametrize("new,cached", [([1], [500]), ([40], [30])])
def test_attention_extreme_scores_and_scales(std, scale, new, cached):
    """Scores far apart: the largest one takes all.  Keys are multiples of one vector, a power of two apart, so that fp32 has them in order."""
    B = _binding()
    latent, rope, heads = 256, 32, 3
    cache = U.Cache(U.blocks_for(new, cached), latent, rope)
    batch = U.Batch(new, cached, cache.n)
    key = U.normal((latent + rope,), 8)
    for p in range(cached[0] + new[0]):
        cache.pool[batch.table[0][p // 16], p % 16] = key * 2.0 ** (p % 7 if p % 31 == 7 else -(p % 5))
    q = key.abs().sign() * key
    q = (q * std).expand(new[0], heads, -1).contiguous()
    ref, tol = cache.attention(batch, q, scale)
    got = U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), scale)
    U.check(got, ref, tol)


@pytest.mark.parametrize("workspace", [True, 0])
def test_attention_scores_that_are_all_minus_infinity_give_zeros(workspace):
    B = _binding()
    cache = U.Cache(40, 128, 32)
    batch = U.Batch([2], [500], cache.n)
    cache.pool[:] = -3e38
    q = torch.full((2, 4, 160), 3e38).bfloat16()
    assert (U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), 1.0, workspace=workspace) == 0).all()


def test_attention_gives_the_same_bits_twice():
    a = _attention(512, 64, 20, [1, 3, 1], [3000, 900, 50])
    b = _attention(512, 64, 20, [1, 3, 1], [3000, 900, 50])
    assert torch.equal(a, b)


def test_pools_beyond_32_bit_offsets():
    """Blocks whose bytes lie beyond 2^32 from the pool's start: append, attention, gather."""
    B = _binding()
    latent, rope, heads, n = 512, 64, 4, 240000            # 4.4 GB
    small = U.Cache(6, latent, rope)
    batch = U.Batch([3], [60], 6)
    q = U.normal((3, heads, latent + rope), 2)
    x, cos_sin = U.normal((3, latent + rope), 3), U.rope_tables(80, rope)
    pool, pool_tol, _, _ = U.append(small, batch, x, None, 0.0, q[..., :rope], q[..., :rope], *cos_sin, 80, False)
    dev = torch.zeros((n, 16, latent + rope), dtype=torch.bfloat16, device="cuda")
    far = n - 6
    dev[far:] = small.pool.cuda()
    small.n = n
    batch.table = [[b + far for b in batch.table[0]]]
    xd, c, s = x.cuda(), cos_sin[0].cuda(), cos_sin[1].cuda()
    B.fp_op_latent_append(small.struct(B, dev), batch.struct(B), xd.data_ptr(), latent + rope, None, 0.0, 3, c.data_ptr(), s.data_ptr(), 80, 0)
    torch.cuda.synchronize()
    U.check(dev[far:], pool, pool_tol)
    now = dev[far:].cpu()
    rows = torch.cat([now[b - far] for b in batch.table[0]])[:63]
    out = [torch.zeros((63, w), dtype=torch.bfloat16, device="cuda") for w in (latent, rope)]
    cu = torch.tensor([0, 63], dtype=torch.int32, device="cuda")
    B.fp_op_latent_gather(small.struct(B, dev), batch.struct(B), cu.data_ptr(), 63, out[0].data_ptr(), out[1].data_ptr())
    got = U.attend(B, small, dev, batch, q.cuda(), 0.05)
    assert torch.equal(torch.cat([o.cpu() for o in out], 1), rows)
    for i in range(3):
        sees = rows[:61 + i].double()
        ref, tol = U.softmax_sum(q[i].double(), sees, sees[:, :latent], 0.05)
        U.check(got[i], ref, tol)


# ---- expanded attention ----

def _expanded(heads, nope, rope, v, new, lens, edit=None, scale=None, std=1.0, **kw):
    B = _binding()
    q = U.normal((sum(new), heads, nope + rope), 1, std)
    kv, kr = U.normal((sum(lens), heads, nope + v), 2), U.normal((sum(lens), rope), 3)
    if edit:
        edit(kv, kr)
    scale = scale or (nope + rope) ** -0.5
    ref, tol = U.expanded(new, lens, q, kv, kr, nope, scale)
    got = U.attend_expanded(B, new, lens, q.cuda(), kv.cuda(), kr.cuda(), nope, scale, **kw)
    U.check(got, ref, tol)
    return got


EXPANDED = [([1], [1]), ([64], [64]), ([65], [65]), ([1, 0, 3], [1, 5, 200]), ([257], [257]), ([40, 300], [40, 333]), ([1] * 70, [3 * i + 1 for i in range(70)])]


@pytest.mark.parametrize("heads,nope,rope,v", [(5, 128, 64, 128), (4, 64, 32, 64), (3, 128, 32, 64), (2, 64, 64, 128), (1, 128, 64, 64),
                                               (2, 64, 32, 128), (9, 128, 32, 128), (2, 64, 64, 64)])
@pytest.mark.parametrize("new,lens", EXPANDED)
def test_expanded_matches_the_definition(heads, nope, rope, v, new, lens):
    _expanded(heads, nope, rope, v, new, lens)


@pytest.mark.parametrize("workspace", [True, 0, "some"])
@pytest.mark.parametrize("heads,new,lens", [(4, [30], [2500]), (3, [1, 100], [1100, 1500]), (2, [3, 0, 260], [0, 4, 1200])])
def test_expanded_of_keys_cut_into_parts(heads, new, lens, workspace):
    B = _binding()
    need = B.fp_op_latent_expanded_attention_workspace_bytes(sum(new), len(new), heads, 128, max(new), max(lens))
    assert need > 0
    _expanded(heads, 128, 64, 128, new, lens, workspace=need // 2 if workspace == "some" else workspace)


def test_expanded_rows_without_keys_are_zero():
    """More queries than keys: the first ones stand before the first position."""
    got = _expanded(2, 64, 32, 64, [5, 3, 300], [2, 0, 40])
    assert (got[:3] == 0).all() and (got[5:8] == 0).all() and (got[8:268] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [5, 64 + 9])
def test_expanded_what_is_not_finite_reaches_only_rows_that_see_it(bad, at):
    def edit(kv, kr):
        kv[69, 1, at] = bad                              # a key's own part, or a value
        kv[100, 0, at] = bad
        kr[130, 3] = bad
    _expanded(3, 64, 32, 64, [40, 90], [70, 90], edit=edit)


def test_expanded_strides_padding_and_rows():
    """Rows of kv inside longer ones, NaN behind the rows that the call has, outputs left alone behind the batch."""
    B = _binding()
    new, lens, heads, nope, rope, v = [3, 70], [50, 90], 2, 64, 32, 64
    t, rows = sum(new), sum(lens)
    q, kv, kr = U.normal((t + 4, heads, 96), 1), U.normal((rows, heads, 128), 2), U.normal((rows, rope), 3)
    ref, tol = U.expanded(new, lens, q, kv, kr, nope, 0.1, t, rows - 7)
    big = torch.full((rows, heads * 128 + 24), math.nan, dtype=torch.bfloat16, device="cuda")
    big[:rows - 7, :heads * 128] = kv[:rows - 7].reshape(rows - 7, -1).cuda()
    krd = torch.full((rows, rope + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    krd[:rows - 7, :rope] = kr[:rows - 7].cuda()
    o = torch.full((t + 4, heads, v + 8), 7.0, dtype=torch.bfloat16, device="cuda")[..., :v]
    o = torch.full((t + 4, heads * v + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    U.attend_expanded(B, new, lens, q.cuda(), big[:, :heads * 128].view(rows, heads, 128), krd[:, :rope], nope, 0.1,
                      o=o[:, :heads * v].view(t + 4, heads, v), tokens=t + 4, rows=rows - 7)
    U.check(o[:t, :heads * v].reshape(t, heads, v), ref[:t], tol[:t])
    assert (o[t:] == 7).all() and (o[:, heads * v:] == 7).all()


@pytest.mark.parametrize("std,scale", [(1e6, 3.0), (1.0, 1e30), (1e-20, 1.0)])
def test_expanded_extreme_scores(std, scale):
    B = _binding()
    key = U.normal((96,), 8)
    kv, kr = U.normal((100, 2, 128), 2), torch.zeros((100, 32)).bfloat16()
    for p in range(100):
        f = 2.0 ** (p % 7 if p % 31 == 7 else -(p % 5))
        kv[p, :, :64], kr[p] = key[:64] * f, key[64:] * f
    q = (key * std).expand(40, 2, -1).contiguous()
    ref, tol = U.expanded([40], [100], q, kv, kr, 64, scale)
    U.check(U.attend_expanded(B, [40], [100], q.cuda(), kv.cuda(), kr.cuda(), 64, scale), ref, tol)


# ---- products per head ----

@pytest.mark.parametrize("n,k", [(512, 128), (128, 512), (8, 8), (64, 256), (136, 40), (256, 64), (24, 1000)])
@pytest.mark.parametrize("m", [1, 15, 16, 17, 64, 65, 257, 400])
@pytest.mark.parametrize("heads", [1, 5])
def test_gemm_heads_matches_the_definition(m, heads, n, k):
    """Heads inside longer rows on both sides; what lies between stays as it was."""
    B = _binding()
    a, w = U.normal((m, heads, k + 16), 1), U.normal((heads, n, k), 2)
    c = torch.full((m, heads, n + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ad, wd = a.cuda(), w.cuda()
    B.fp_op_gemm_heads(ad.data_ptr(), ad.stride(0), ad.stride(1), wd.data_ptr(), wd.stride(0), c.data_ptr(), c.stride(0), c.stride(1), m, heads, n, k)
    torch.cuda.synchronize()
    x, y = a[..., :k].double().transpose(0, 1), w.double().transpose(1, 2).contiguous()
    ref, size = (x @ y).transpose(0, 1), (x.abs() @ y.abs()).transpose(0, 1)
    U.check(c[..., :n], ref, U.HALF_BF16 * ref.abs() + (k + 1) * U.HALF_FP32 * size)
    assert (c[..., n:] == 7).all()


@pytest.mark.parametrize("m,heads,n,k", [(450, 33, 512, 128), (300, 50, 136, 512), (700, 24, 264, 256), (1000, 16, 520, 64), (3600, 4, 64, 256), (7200, 2, 8, 128)])
def test_gemm_heads_of_many_tokens(m, heads, n, k):
    """Weights in LDS: more outputs than fit, outputs and tokens that end inside a round."""
    test_gemm_heads_matches_the_definition(m, heads, n, k)


def test_gemm_heads_of_a_slice_of_the_weights():
    """W_uv as rows N .. N+V-1 of every head of the up projection: a head stride beyond the head's own numbers; NaN elsewhere is not read."""
    B = _binding()
    heads, nope, v, latent, m = 3, 64, 128, 256, 20
    full = torch.full((heads, nope + v, latent), math.nan, dtype=torch.bfloat16, device="cuda")
    w, a = U.normal((heads, v, latent), 1), U.normal((m, heads, latent), 2)
    full[:, nope:] = w.cuda()
    c, ad = torch.zeros((m, heads, v), dtype=torch.bfloat16, device="cuda"), a.cuda()
    B.fp_op_gemm_heads(ad.data_ptr(), ad.stride(0), ad.stride(1), full[:, nope:].data_ptr(), full.stride(0), c.data_ptr(), c.stride(0), c.stride(1),
                       m, heads, v, latent)
    torch.cuda.synchronize()
    x, y = a.double().transpose(0, 1), w.double().transpose(1, 2).contiguous()
    ref, size = (x @ y).transpose(0, 1), (x.abs() @ y.abs()).transpose(0, 1)
    U.check(c, ref, U.HALF_BF16 * ref.abs() + (latent + 1) * U.HALF_FP32 * size)


@pytest.mark.parametrize("workspace", [True, 0])
@pytest.mark.parametrize("heads,new,lens", [
    (40, [257, 3, 300, 0, 256, 90], [257, 1500, 700, 4, 256, 30]),      # tiles of unlike lengths, queries before the first key
    (48, [70] * 5, [70] * 5),                                           # all alike
    (90, [1, 300], [4300, 300]),                                        # more steps than a wave has lanes
    (40, [20, 1, 33, 2, 64, 9, 17, 5], [20, 700, 40, 90, 64, 1, 300, 5]),           # as many sequences as are ordered, and one more
    (40, [20, 1, 33, 2, 64, 9, 17, 5, 8], [20, 700, 40, 90, 64, 1, 300, 5, 8]),
])
def test_expanded_batches_whose_tiles_start_by_their_steps(heads, new, lens, workspace):
    """More workgroups than CUs, so that the order of the tiles is taken from the lengths."""
    assert ((sum(new) - len(new)) // 256 + len(new)) * heads > 256
    _expanded(heads, 64, 32, 64, new, lens, workspace=workspace)
