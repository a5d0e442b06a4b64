"""Calls of latent attention's operators that are refused, without a GPU: nothing is launched, and the message says what is wrong."""
import pytest

GOOD = 1 << 20                     # an address that is aligned and never read


def _call(name, **change):
    from paper_2602_16603_amd import binding as B
    c = dict(pool=GOOD, num_blocks=8, latent_dim=512, rope_dim=64, n_seqs=2, max_blocks=4, cu=GOOD, cached=GOOD, table=GOOD)
    calls = {
        "append": dict(latent=GOOD, latent_stride=576, gain=GOOD, eps=1e-6, n_tokens=3, cos=GOOD, sin=GOOD, max_position=64, pairing=0, heads=4,
                       q=GOOD, q_stride=4 * 192, q_head_stride=192, q_out=2 * GOOD, q_out_stride=4 * 576, q_out_head_stride=576),
        "attention": dict(q=GOOD, q_stride=4 * 576, o=GOOD, o_stride=4 * 512, n_tokens=3, heads=4, scale=0.1, max_new=2, max_len=64, ws=0, ws_bytes=0),
        "gather": dict(cu_out=GOOD, n_rows=5, latent_out=GOOD, rope_out=GOOD),
        "expanded": dict(cu_q=GOOD, cu_kv=GOOD, n=2, q=GOOD, q_stride=4 * 192, kv=GOOD, kv_stride=4 * 256, kr=GOOD, kr_stride=64, o=GOOD,
                         o_stride=4 * 128, n_tokens=3, n_rows=9, heads=4, nope=128, rope=64, v=128, scale=0.1, max_new=2, max_len=64, ws=0, ws_bytes=0),
        "heads": dict(a=GOOD, a_stride=4 * 192, a_head=192, w=GOOD, w_head=512 * 128, c=GOOD, c_stride=4 * 576, c_head=576, m=3, heads=4, n=512, k=128),
    }
    a = calls[name]
    for key, value in change.items():
        assert key in a or key in c, key
        (a if key in a else c)[key] = value
    cache = None if c["num_blocks"] == "null" else B.fp_latent_cache(c["pool"], c["num_blocks"], c["latent_dim"], c["rope_dim"])
    batch = None if c["n_seqs"] == "null" else B.fp_latent_batch(c["n_seqs"], c["max_blocks"], c["cu"], c["cached"], c["table"])
    if name == "append":
        B.fp_op_latent_append(cache, batch, a["latent"], a["latent_stride"], a["gain"], a["eps"], a["n_tokens"], a["cos"], a["sin"], a["max_position"],
                              a["pairing"], a["heads"], a["q"], a["q_stride"], a["q_head_stride"], a["q_out"], a["q_out_stride"], a["q_out_head_stride"])
    elif name == "attention":
        B.fp_op_latent_attention(cache, batch, a["q"], a["q_stride"], a["o"], a["o_stride"], a["n_tokens"], a["heads"], a["scale"], a["max_new"],
                                 a["max_len"], a["ws"], a["ws_bytes"])
    elif name == "gather":
        B.fp_op_latent_gather(cache, batch, *a.values())
    elif name == "expanded":
        B.fp_op_latent_expanded_attention(*a.values())
    else:
        B.fp_op_gemm_heads(*a.values())


CACHE = [dict(pool=0), dict(pool=GOOD + 8), dict(num_blocks=0), dict(num_blocks=1 << 31), dict(num_blocks="null"), dict(latent_dim=384), dict(latent_dim=0),
         dict(rope_dim=48), dict(n_seqs="null"), dict(n_seqs=-1), dict(max_blocks=0), dict(max_blocks=(1 << 26) + 1), dict(table=0), dict(table=GOOD + 2)]
LENGTHS = [dict(cu=0), dict(cached=0), dict(cu=GOOD + 1), dict(cached=GOOD + 2)]
WORK = [dict(ws_bytes=-1), dict(ws_bytes=256), dict(ws=GOOD + 128, ws_bytes=512)]
SCALE = [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.4e38)]
HINTS = [dict(max_new=0), dict(max_len=0), dict(max_new=-1)]
REFUSED = [("append", c) for c in CACHE + LENGTHS + [
    dict(latent=0), dict(latent=GOOD + 4), dict(latent_stride=568), dict(latent_stride=580), dict(gain=GOOD + 8), dict(eps=-1.0), dict(eps=float("nan")),
    dict(n_tokens=-1), dict(n_tokens=1 << 24), dict(cos=0), dict(sin=GOOD + 4), dict(max_position=0), dict(pairing=2), dict(pairing=-1), dict(heads=-1),
    dict(heads=65537), dict(q=0), dict(q=GOOD + 2), dict(q_out=0), dict(q_stride=3 * 192), dict(q_stride=4 * 192 + 4), dict(q_head_stride=56),
    dict(q_out_head_stride=60), dict(q_out_stride=576), dict(q_head_stride=1 << 24, q_stride=1 << 30), dict(q_out=GOOD)]]
REFUSED += [("attention", c) for c in CACHE + LENGTHS + WORK + SCALE + HINTS + [
    dict(q=0), dict(q=GOOD + 8), dict(o=0), dict(o=GOOD + 8), dict(q_stride=4 * 576 - 8), dict(q_stride=4 * 576 + 4), dict(o_stride=4 * 512 - 8),
    dict(n_tokens=-1), dict(n_tokens=1 << 24), dict(heads=0), dict(heads=65537), dict(heads=16384, n_tokens=8192, q_stride=1 << 30, o_stride=1 << 30),
    dict(heads=65536, n_tokens=64, n_seqs=64, q_stride=1 << 30, o_stride=1 << 30)]]
REFUSED += [("gather", c) for c in CACHE + [dict(cu_out=0), dict(cu_out=GOOD + 2), dict(n_rows=-1), dict(n_rows=1 << 29), dict(latent_out=0),
                                            dict(latent_out=GOOD + 8), dict(rope_out=0)]]
REFUSED += [("expanded", c) for c in WORK + SCALE + HINTS + [
    dict(cu_q=0), dict(cu_kv=0), dict(cu_kv=GOOD + 1), dict(n=-1), dict(q=0), dict(kv=GOOD + 8), dict(kr=0), dict(o=GOOD + 8), dict(q_stride=760),
    dict(kv_stride=1016), dict(kv_stride=1028), dict(kv_stride=(1 << 23) + 8), dict(kr_stride=56), dict(kr_stride=(1 << 23) + 8), dict(o_stride=504),
    dict(n_tokens=-1), dict(n_tokens=1 << 24), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(heads=0), dict(nope=96), dict(rope=128), dict(v=192)]]
REFUSED += [("heads", c) for c in [
    dict(a=0), dict(a=GOOD + 8), dict(w=0), dict(c=0), dict(c=GOOD + 2), dict(m=-1), dict(m=1 << 31), dict(heads=0), dict(n=0), dict(n=12), dict(k=0), dict(k=4),
    dict(k=(1 << 20) + 8), dict(n=(1 << 20) + 8), dict(a_head=120), dict(a_stride=3 * 192 + 120), dict(a_stride=769), dict(c_head=504), dict(c_stride=3 * 576 + 504),
    dict(w_head=512 * 128 - 8), dict(m=1 << 30, a_stride=1 << 20, c_stride=1 << 20)]]


@pytest.mark.parametrize("name,change", REFUSED)
def test_refused(name, change):
    from paper_2602_16603_amd import binding as B
    with pytest.raises(B.FlowPrefillError) as e:
        _call(name, **change)
    assert e.value.status == B.FP_ERR_INVALID and str(e.value).split(": ", 2)[2]


@pytest.mark.parametrize("name,change", [
    ("append", dict(n_tokens=0)), ("append", dict(n_seqs=0)), ("append", dict(n_tokens=0, heads=0, q=0, q_out=0)), ("attention", dict(n_tokens=0)),
    ("attention", dict(n_seqs=0, cu=0, cached=0, table=0)), ("attention", dict(n_tokens=0, scale=2.3e38)), ("gather", dict(n_rows=0)), ("gather", dict(n_seqs=0)),
    ("expanded", dict(n_tokens=0)), ("expanded", dict(n=0)), ("heads", dict(m=0)),
])
def test_empty_calls_launch_nothing(name, change):
    _call(name, **change)


def test_workspace_of_calls_that_are_refused_is_zero():
    from paper_2602_16603_amd import binding as B
    assert B.fp_op_latent_attention_workspace_bytes(1, 1, 16, 512, 64, 1, 30000) > 0
    for bad in ((0, 1, 16, 512, 64, 1, 100), (1, 0, 16, 512, 64, 1, 100), (1, 1, 0, 512, 64, 1, 100), (1, 1, 16, 384, 64, 1, 100),
                (1, 1, 16, 512, 64, 0, 100), (1, 1, 16, 512, 64, 1, -1), (1 << 24, 1, 16, 512, 64, 1, 100)):
        assert B.fp_op_latent_attention_workspace_bytes(*bad) == 0
    assert B.fp_op_latent_expanded_attention_workspace_bytes(1, 1, 16, 128, 1, 30000) > 0
    for bad in ((0, 1, 16, 128, 1, 100), (1, 1, 16, 96, 1, 100), (1, 1, 65537, 128, 1, 100), (1, 1, 16, 128, 1, 0)):
        assert B.fp_op_latent_expanded_attention_workspace_bytes(*bad) == 0


def test_gather_of_more_sequences_than_a_launch_holds_is_refused():
    """128 threads for a slot of 16 rows, a slot for every sequence: 2^25 - 1 slots round up to 2^32 threads."""
    from paper_2602_16603_amd import binding as B
    for rows, seqs in ((1, (1 << 25) - 1), (16, (1 << 25) - 2), (33, (1 << 25) - 3)):
        with pytest.raises(B.FlowPrefillError) as e:
            _call("gather", n_rows=rows, n_seqs=seqs)
        assert e.value.status == B.FP_ERR_INVALID
