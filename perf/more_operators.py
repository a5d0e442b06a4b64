"""The operators of latent attention, as timed cases.

A model with latent attention caches one vector a token for all its heads: a latent of R numbers, normalised, and P numbers of a
rotated key that the heads share.  A paged pool holds them as rows [R | P] in bf16, 16 tokens to a block.  Per head, a key is
[W_uk latent | rotated part] (N + P numbers) and a value W_uv latent (V numbers).  The operators:
  append    normalises the latents of new tokens, rotates the keys' and the queries' parts by position, writes the pages
  attention absorbed form: queries that went through W_uk^T (R + P numbers a head) over the pages themselves; the outputs are sums of
            latents (R numbers a head)
  heads     a product per head: W_uk^T into the queries before, W_uv onto the outputs after the absorbed form
  gather    the sequences' rows out of the pages, contiguous: what the expanded form's keys and values are projected from
  expanded  attention over keys and values projected for every head (N + P and V numbers), causal, packed sequences
A batch is described as for the 8-bit cache: cu_seqlens, the tokens that each sequence has in the cache already (negative: an idle
slot), its row of the block table (an entry outside the pool: a block that is not there).
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
EPS = 1e-6
THETA = 10000.0
WORKSPACE = 96 << 20             # bytes of scratch that the program keeps for its attention calls
# heads, R, P, N, V
SHAPES = {"20": (20, 512, 64, 128, 128), "32": (32, 512, 64, 128, 128), "128": (128, 512, 64, 128, 128), "40": (40, 256, 32, 64, 64),
          "tiny": (4, 128, 32, 64, 64)}


def _case(name, kind, shape, new, cached, interleaved=False, evicted=0, down=False):
    """`new`, `cached`: tokens per sequence; `evicted`: blocks that each sequence has given up, from its second block on; `down`: the
    product after the attention, not the one before it."""
    return {"name": name, "kind": kind, "shape": shape, "new": ",".join(map(str, new)), "cached": ",".join(map(str, cached)),
            "interleaved": interleaved, "evicted": evicted, "down": down}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some(seed, n, lo, hi):
    rng = random.Random(seed)
    return [_log_int(rng, lo, hi) for _ in range(n)]


def listed():
    return [
        # A decode step of a batch, one token each at odd places of their blocks, two slots idle: launch latency.
        _case("append_step_32", "append", "128", [1] * 32, _some(1, 30, 16, 8191) + [-1, -1], True),
        # The benchmark's prompt length: the bytes of latents and queries.
        _case("append_prompt_8192", "append", "20", [8192], [0], True),
        # One token of a tiny stack: latency.
        _case("attend_step_tiny", "attention", "tiny", [1], [200]),
        # One token of many heads behind a long prompt: few rows, a long axis.
        _case("attend_step_long", "attention", "128", [1], [32767]),
        # A decode step of a batch of ragged lengths, four slots idle, old blocks evicted: the cache's bytes.
        _case("attend_step_64", "attention", "20", [1] * 64, _some(2, 60, 512, 16384) + [-1] * 4, evicted=16),
        # Chunked prefill in the absorbed form: the last 512-token chunk of a 16384-token prompt.
        _case("attend_chunk_512_of_16384", "attention", "20", [512], [15872]),
        # A decode step's queries through W_uk^T: the weights' bytes.
        _case("heads_up_step_64", "heads", "128", [64], [0]),
        # A packed prefill batch's outputs through W_uv: the activations' bytes.
        _case("heads_down_4096", "heads", "32", [4096], [0], down=True),
        # The rows of the mean text request, and of a packed batch with long prefixes.
        _case("gather_777", "gather", "20", [777], [0]),
        _case("gather_packed", "gather", "20", [1024, 512, 2048, 333], [15360, 20000, 1000, 30001]),
        # A packed prefill batch, some of its prompts continued behind a prefix.
        _case("expand_packed", "expanded", "32", [1213, 64, 590, 2002, 227], [0, 37, 0, 515, 1600]),
        # The benchmark's prompt length.
        _case("expand_prompt_8192", "expanded", "20", [8192], [0]),
    ]


def _slots(rng, n, lo, hi):
    """Cached lengths of a decode batch; now and then a slot is idle, never the first."""
    return [-1 if s and rng.random() < 0.05 else _log_int(rng, lo, hi) for s in range(n)]


def draw(rng):
    kind = rng.choice(["append_step", "append_prompts", "step", "step", "step", "long", "draft", "chunk", "heads", "heads", "gather",
                       "expand_prompts", "expand_chunk"])
    shape = rng.choice(["20", "20", "32", "40", "128", "128", "tiny"])
    wide = shape == "128"
    if kind == "append_step":
        n = _log_int(rng, 1, 128)
        return _case("", "append", shape, [1] * n, _slots(rng, n, 1, 16000), rng.random() < 0.5)
    if kind == "append_prompts":
        n = rng.randint(1, 8)
        return _case("", "append", shape, [_log_int(rng, 16, 256 if wide else 1000) for _ in range(n)],
                     [rng.choice([0, _log_int(rng, 1, 8000)]) for _ in range(n)], rng.random() < 0.5)
    if kind == "step":
        n = _log_int(rng, 1, 32 if wide else 96)
        return _case("", "attention", shape, [1] * n, _slots(rng, n, 64, rng.choice([1000, 4000, 12000])))
    if kind == "long":
        return _case("", "attention", shape, [1], [_log_int(rng, 4000, 60000)], evicted=rng.choice([0, 0, 100]))
    if kind == "draft":
        n = rng.randint(1, 8 if wide else 32)
        return _case("", "attention", shape, [rng.randint(1, 8) for _ in range(n)], [_log_int(rng, 64, 6000) for _ in range(n)])
    if kind == "chunk":
        return _case("", "attention", shape, [_log_int(rng, 16, 64 if wide else 256)], [_log_int(rng, 512, 15000)])
    if kind == "heads":
        return _case("", "heads", shape, [_log_int(rng, 1, 900 if wide else 4096)], [0], down=rng.random() < 0.5)
    if kind == "gather":
        n = rng.randint(1, 5)
        return _case("", "gather", shape, [_log_int(rng, 1, 2000) for _ in range(n)], [_log_int(rng, 16, 12000) for _ in range(n)])
    if kind == "expand_prompts":
        return _case("", "expanded", shape, [_log_int(rng, 16, 1100 if wide else 2400) for _ in range(rng.randint(1, 4))], [0])
    return _case("", "expanded", shape, [_log_int(rng, 16, 128 if wide else 1000)], [_log_int(rng, 256, 8000)])


def _ints(case):
    new = [int(n) for n in case["new"].split(",")]
    cached = [int(n) for n in case["cached"].split(",")]
    return new, cached + [0] * (len(new) - len(cached))


def prepare(case, seed):
    heads, lat, rot, nope, val = SHAPES[case["shape"]]
    new, cached = _ints(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*size):
        return torch.randn(size, generator=g, device="cuda").bfloat16()

    tokens = sum(new)
    st = {"case": case, "heads": heads, "lat": lat, "rot": rot, "nope": nope, "val": val, "tokens": tokens, "scale": (nope + rot) ** -0.5}
    if case["kind"] == "heads":
        n, k = (val, lat) if case["down"] else (lat, nope)
        # Rows of W_uk^T and W_uv, about as large as trained ones; a query or an output of R + P or N + P numbers has a tail that the
        # product leaves alone.
        st["w"] = (torch.randn((heads, n, k), generator=g, device="cuda") * k ** -0.5).bfloat16()
        st["a"] = normal(tokens, heads, k if case["down"] else k + rot)
        st["c"] = normal(tokens, heads, n if case["down"] else n + rot)
        return st
    total = [max(c, 0) + n if c >= 0 else 0 for n, c in zip(new, cached)]
    st.update(max_new=max(new), max_len=max(total), cu=torch.tensor([0] + new, device="cuda").cumsum(0).int(),
              cached=torch.tensor(cached, dtype=torch.int32, device="cuda"), cu_all=torch.tensor([0] + total, device="cuda").cumsum(0).int())
    if case["kind"] == "expanded":
        rows = sum(total)
        st["q"] = normal(tokens, heads, nope + rot)
        st["kv"] = normal(rows, heads, nope + val)
        st["k_rope"] = normal(rows, rot)
        st["o"] = torch.empty((tokens, heads, val), dtype=torch.bfloat16, device="cuda")
        st["ws"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        return st
    need = [-(-t // BLOCK) for t in total]
    blocks = sum(need) + 32
    # Blocks of a pool that has been in use lie scattered over it.
    perm = torch.randperm(blocks, generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((len(new), max(need + [1])), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, nb in enumerate(need):
        table[s, :nb] = perm[at:at + nb]
        table[s, 1:1 + min(case["evicted"], max(0, nb - 4))] = -1
        at += nb
    st["table"] = table
    st["pool"] = normal(blocks, BLOCK, lat + rot)
    if case["kind"] == "append":
        # Latents as a projection leaves them, before their norm: channels of different sizes.
        st["x"] = (torch.randn((tokens, lat + rot), generator=g, device="cuda") *
                   torch.exp(0.5 * torch.randn((lat + rot,), generator=g, device="cuda"))).bfloat16()
        st["gain"] = (1 + 0.1 * torch.randn((lat,), generator=g, device="cuda")).bfloat16()
        st["q"] = normal(tokens, heads, nope + rot)
        st["q_out"] = torch.zeros((tokens, heads, lat + rot), dtype=torch.bfloat16, device="cuda")
        angle = torch.arange(max(total), device="cuda", dtype=torch.float64)[:, None] * THETA ** (
            -torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
    elif case["kind"] == "attention":
        st["q"] = normal(tokens, heads, lat + rot)
        st["o"] = torch.empty((tokens, heads, lat), dtype=torch.bfloat16, device="cuda")
        st["ws"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    else:
        st["latent_out"] = torch.empty((sum(total), lat), dtype=torch.bfloat16, device="cuda")
        st["rope_out"] = torch.empty((sum(total), rot), dtype=torch.bfloat16, device="cuda")
    return st


def run(st):
    kind = st["case"]["kind"]
    if own:
        _call(st)
    else:
        {"append": _append, "attention": _attend, "heads": _heads, "gather": _gather, "expanded": _expanded}[kind](st)
    if kind == "append":
        return {"pool": st["pool"], "q": st["q_out"]}
    if kind == "gather":
        return {"latent": st["latent_out"], "rope": st["rope_out"]}
    return st["c"] if kind == "heads" else st["o"]


# ---- the framework's operators ----

def _call(st):
    from paper_2602_16603_amd import binding as B
    kind, heads, lat, rot, nope, tokens = st["case"]["kind"], st["heads"], st["lat"], st["rot"], st["nope"], st["tokens"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "heads":
        a, w, c = st["a"], st["w"], st["c"]
        B.fp_op_gemm_heads(a.data_ptr(), a.stride(0), a.stride(1), w.data_ptr(), w.stride(0), c.data_ptr(), c.stride(0), c.stride(1),
                           tokens, heads, w.shape[1], w.shape[2], stream)
        return
    if kind == "expanded":
        q, kv, kr, o = st["q"], st["kv"], st["k_rope"], st["o"]
        B.fp_op_latent_expanded_attention(st["cu"].data_ptr(), st["cu_all"].data_ptr(), st["cached"].shape[0], q.data_ptr(), q.stride(0),
                                          kv.data_ptr(), kv.stride(0), kr.data_ptr(), kr.stride(0), o.data_ptr(), o.stride(0), tokens,
                                          kv.shape[0], heads, nope, rot, st["val"], st["scale"], st["max_new"], st["max_len"],
                                          st["ws"].data_ptr(), WORKSPACE, stream)
        return
    table = st["table"]
    cache = B.fp_latent_cache(st["pool"].data_ptr(), st["pool"].shape[0], lat, rot)
    batch = B.fp_latent_batch(table.shape[0], table.shape[1], st["cu"].data_ptr(), st["cached"].data_ptr(), table.data_ptr())
    if kind == "append":
        x, q, q_out = st["x"], st["q"], st["q_out"]
        pairing = B.FP_ROPE_INTERLEAVED if st["case"]["interleaved"] else B.FP_ROPE_HALF
        B.fp_op_latent_append(cache, batch, x.data_ptr(), x.stride(0), st["gain"].data_ptr(), EPS, tokens, st["cos"].data_ptr(),
                              st["sin"].data_ptr(), st["cos"].shape[0], pairing, heads, q[..., nope:].data_ptr(), q.stride(0), q.stride(1),
                              q_out[..., lat:].data_ptr(), q_out.stride(0), q_out.stride(1), stream)
    elif kind == "attention":
        q, o = st["q"], st["o"]
        B.fp_op_latent_attention(cache, batch, q.data_ptr(), q.stride(0), o.data_ptr(), o.stride(0), tokens, heads, st["scale"],
                                 st["max_new"], st["max_len"], st["ws"].data_ptr(), WORKSPACE, stream)
    else:
        B.fp_op_latent_gather(cache, batch, st["cu_all"].data_ptr(), st["latent_out"].shape[0], st["latent_out"].data_ptr(),
                              st["rope_out"].data_ptr(), stream)


# ---- plain forms ----

def _rotate(x, cos, sin, interleaved):
    """Last axis in pairs, turned by the tables' angles; in 64 bits, as the angles of far positions need it."""
    half = x.shape[-1] // 2
    x, c, s = x.double(), cos.double(), sin.double()
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _append(st):
    lat, nope, tokens = st["lat"], st["nope"], st["tokens"]
    cu, cached = st["cu"].long(), st["cached"].long()
    row = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(cu[1:], row, right=True)
    pos = cached[seq] + row - cu[seq]
    busy = cached[seq] >= 0
    row, seq, pos = row[busy], seq[busy], pos[busy]
    cos, sin = st["cos"][pos], st["sin"][pos]
    x = st["x"][row].float()
    c = x[:, :lat]
    c = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS) * st["gain"].float()
    k = _rotate(x[:, lat:], cos, sin, st["case"]["interleaved"])
    st["q_out"][row, :, lat:] = _rotate(st["q"][row, :, nope:], cos[:, None], sin[:, None], st["case"]["interleaved"]).bfloat16()
    blk = st["table"][seq, pos // BLOCK].long()
    there = (blk >= 0) & (blk < st["pool"].shape[0])
    st["pool"][blk[there], (pos % BLOCK)[there]] = torch.cat([c.bfloat16(), k.bfloat16()], -1)[there]


def _attend(st):
    heads, lat, rot, tokens = st["heads"], st["lat"], st["rot"], st["tokens"]
    cu, cached, table = st["cu"].long(), st["cached"].long(), st["table"].long()
    there = (table >= 0) & (table < st["pool"].shape[0])
    seqs, nb = table.shape
    # Padded to the batch's longest: keys [S, L, R + P], queries [S, new * heads, R + P].
    k = st["pool"][torch.where(there, table, 0)].float().reshape(seqs, nb * BLOCK, lat + rot)
    i = torch.arange(st["max_new"], device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=tokens - 1)
    q = st["q"][rows].float().reshape(seqs, -1, lat + rot)
    pos = torch.where(cached[:, None] >= 0, cached[:, None] + i, -1)
    sees = (torch.arange(nb * BLOCK, device="cuda") <= pos[..., None]) & there.repeat_interleave(BLOCK, 1)[:, None]
    p = (q @ k.transpose(1, 2)).mul_(st["scale"]).masked_fill_(~sees.repeat_interleave(heads, 1), -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, (p @ k[..., :lat]) / total, 0.0).view(seqs, st["max_new"], heads, lat)
    row = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(cu[1:], row, right=True)
    st["o"].copy_(o[seq, row - cu[seq]])


def _heads(st):
    n, k = st["w"].shape[1:]
    prod = st["a"][..., :k].float().transpose(0, 1) @ st["w"].float().transpose(1, 2)
    st["c"][..., :n] = prod.transpose(0, 1).bfloat16()


def _gather(st):
    cu = st["cu_all"].long()
    row = torch.arange(st["latent_out"].shape[0], device="cuda")
    seq = torch.searchsorted(cu[1:], row, right=True)
    pos = row - cu[seq]
    x = st["pool"][st["table"][seq, pos // BLOCK].long(), pos % BLOCK]
    st["latent_out"].copy_(x[:, :st["lat"]])
    st["rope_out"].copy_(x[:, st["lat"]:])


def _expanded(st):
    nope, heads = st["nope"], st["heads"]
    new, cached = _ints(st["case"])
    lo = at = 0
    for n, c in zip(new, cached):
        rows = c + n
        kv, q = st["kv"][at:at + rows].float().transpose(0, 1), st["q"][lo:lo + n].float().transpose(0, 1)
        k = torch.cat([kv[..., :nope], st["k_rope"][at:at + rows].float().expand(heads, -1, -1)], -1)
        p = (q @ k.transpose(1, 2)).mul_(st["scale"])
        p.masked_fill_(torch.arange(rows, device="cuda") > c + torch.arange(n, device="cuda")[:, None], -math.inf)
        p = p.sub_(p.amax(-1, keepdim=True)).exp_()
        st["o"][lo:lo + n] = ((p @ kv[..., nope:]) / p.sum(-1, keepdim=True)).transpose(0, 1).bfloat16()
        lo, at = lo + n, at + rows


# ---- what a pass cannot do without ----

def work(case):
    heads, lat, rot, nope, val = SHAPES[case["shape"]]
    new, cached = _ints(case)
    busy = [(n, c) for n, c in zip(new, cached) if c >= 0]
    t, rows = sum(n for n, _ in busy), sum(n + c for n, c in busy)
    if case["kind"] == "append":
        return {"bytes": 4 * t * (lat + rot + heads * rot) + 2 * lat + 4 * t * rot, "flops": t * (4 * lat + 3 * rot * (heads + 1))}
    if case["kind"] == "heads":
        n, k = (val, lat) if case["down"] else (lat, nope)
        return {"bytes": 2 * heads * (t * (n + k) + n * k), "flops": 2 * heads * t * n * k}
    if case["kind"] == "gather":
        return {"bytes": 4 * rows * (lat + rot) + rows // BLOCK * 4, "flops": 0}
    if case["kind"] == "expanded":
        pairs = sum(n * c + n * (n + 1) // 2 for n, c in busy)
        return {"bytes": 2 * (t * heads * (nope + rot + val) + rows * (heads * (nope + val) + rot)),
                "flops": 2 * heads * (nope + rot + val) * pairs}
    gone = [BLOCK * min(case["evicted"], max(0, -(-(c + n) // BLOCK) - 4)) for n, c in busy]
    keys = sum(c + n - d for (n, c), d in zip(busy, gone))
    pairs = sum(n * (c - d) + n * (n + 1) // 2 for (n, c), d in zip(busy, gone))
    return {"bytes": 2 * (t * heads * (2 * lat + rot) + keys * (lat + rot)), "flops": 2 * heads * (2 * lat + rot) * pairs}


# ---- the same in 64 bits ----

def _turn(x, cos, sin, interleaved):
    """x [n, heads, P] as complex numbers times the unit numbers of the tables [n, P/2]."""
    n, h, p = x.shape
    pairs = x.double().reshape(n, h, p // 2, 2) if interleaved else x.double().reshape(n, h, 2, p // 2).transpose(2, 3)
    z = torch.view_as_complex(pairs.contiguous()) * torch.complex(cos.double(), sin.double())[:, None]
    out = torch.view_as_real(z)
    return (out if interleaved else out.transpose(2, 3)).reshape(n, h, p)


def exact(case, seed):
    st = prepare(case, seed)
    heads, lat, rot, nope, val = SHAPES[case["shape"]]
    new, cached = _ints(case)
    if case["kind"] == "heads":
        out, k = st["c"].double(), st["w"].shape[2]
        for h in range(heads):
            out[:, h, :st["w"].shape[1]] = torch.mm(st["a"][:, h, :k].double(), st["w"][h].double().t())
        return out
    if case["kind"] == "expanded":
        out = torch.zeros(st["o"].shape, dtype=torch.float64, device="cuda")
        lo = at = 0
        for n, c in zip(new, cached):
            hidden = torch.ones((n, c + n), device="cuda").triu(c + 1).bool()
            for h in range(heads):
                q, kv = st["q"][lo:lo + n, h].double(), st["kv"][at:at + c + n, h].double()
                w = q[:, :nope] @ kv[:, :nope].t() + q[:, nope:] @ st["k_rope"][at:at + c + n].double().t()
                out[lo:lo + n, h] = torch.softmax((w / math.sqrt(nope + rot)).masked_fill(hidden, -math.inf), -1) @ kv[:, nope:]
            lo, at = lo + n, at + c + n
        return out
    table = st["table"].tolist()
    if case["kind"] == "gather":
        rows = [st["pool"][table[s][:-(-(c + n) // BLOCK)]].reshape(-1, lat + rot)[:c + n] for s, (n, c) in enumerate(zip(new, cached))]
        rows = torch.cat(rows).double()
        return {"latent": rows[:, :lat].contiguous(), "rope": rows[:, lat:].contiguous()}
    lo = 0
    if case["kind"] == "attention":
        out = torch.zeros(st["o"].shape, dtype=torch.float64, device="cuda")
        for s, (n, c) in enumerate(zip(new, cached)):
            have = [b for b, blk in enumerate(table[s][:-(-(c + n) // BLOCK)]) if blk >= 0] if c >= 0 else []
            if have:
                key = (torch.tensor(have, device="cuda")[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).reshape(-1)
                rows = st["pool"][torch.tensor([table[s][b] for b in have], device="cuda")].reshape(-1, lat + rot).double()
                hidden = key > c + torch.arange(n, device="cuda")[:, None]
                rows[key >= c + n] = 0
                for h in range(heads) if n > 1 else [slice(None)]:
                    q = st["q"][lo:lo + n, h].double()
                    w = (q @ rows.t() / math.sqrt(nope + rot)).masked_fill(hidden, -math.inf)
                    out[lo:lo + n, h] = torch.softmax(w, -1) @ rows[:, :lat]
            lo += n
        return out
    res = {"pool": st["pool"].double(), "q": st["q_out"].double()}
    for s, (n, c) in enumerate(zip(new, cached)):
        if c >= 0:
            x, cos, sin = st["x"][lo:lo + n].double(), st["cos"][c:c + n], st["sin"][c:c + n]
            z = x[:, :lat]
            z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / lat + EPS) * st["gain"].double()
            k = _turn(x[:, None, lat:], cos, sin, case["interleaved"])[:, 0]
            pos = torch.arange(c, c + n, device="cuda")
            res["pool"][st["table"][s].long()[pos // BLOCK], pos % BLOCK] = torch.cat([z, k], -1)
            res["q"][lo:lo + n, :, lat:] = _turn(st["q"][lo:lo + n, :, nope:], cos, sin, case["interleaved"])
        lo += n
    return res
