"""The 8-bit cache's host side, without a GPU: how its operators cut their work (csrc/kv8_plan.h, built for the CPU), and the calls
that its entry points refuse."""
import math
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("kv8") / "dump")
    subprocess.run([cxx, "-std=c++17", "-O2", os.path.join(ROOT, "tests", "host", "kv8_plan_dump.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, l)) for l in lines) + "\n", stdout=subprocess.PIPE, text=True,
                             check=True, timeout=300).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]
    return run


def _batches(count):
    rng = random.Random(7)
    for _ in range(count):
        yield [rng.choice([0, 1, 1, 2, 15, 16, 17, 63, 64, 255, 256, 257, rng.randint(0, 3000)]) for _ in range(rng.randint(1, 40))]


@pytest.mark.parametrize("mult,per,extra", [(1, 16, 2), (4, 16, 1), (5, 32, 1), (8, 256, 1), (1, 1, 0)])
def test_every_row_has_a_slot_of_its_sequence(plan, mult, per, extra):
    """A slot's sequence is found as the kernels find it; the rows a sequence needs (with `extra` = 2: in blocks that its tokens
    may begin anywhere in) are all within its own slots, and the launch has them all."""
    for lengths in _batches(60):
        cu = [0]
        for n in lengths:
            cu.append(cu[-1] + n)
        bases = [v for v, in plan([("slot", c * mult, s, per, extra) for s, c in enumerate(cu)])]
        total, = plan([("slot", cu[-1] * mult, len(lengths), per, extra)])[0]
        assert bases[-1] == total and (extra == 0 or all(a < b for a, b in zip(bases, bases[1:])))
        for s, n in enumerate(lengths):
            for begin in ((0, 1, 7, 15) if extra == 2 else (0,)):
                need = -(-(n * mult + begin) // per) if n else 0
                for slot in range(bases[s], bases[s] + need):
                    owner = sum(b <= slot for b in bases[:-1]) - 1
                    assert owner == s and slot < total, (lengths, s, slot)


def test_parts_and_shares_stay_within_the_workspace(plan):
    rng = random.Random(8)
    calls = []
    for _ in range(3000):
        hkv = rng.choice([1, 2, 4, 8, 5, 1000])
        seqs = rng.choice([1, 2, 16, 64, 500])
        new = rng.choice([1, 1, 2, 5, 40, 512, 9000])
        calls.append(("plan", seqs * new, seqs, hkv * rng.choice([1, 4, 5, 8]), hkv, rng.choice([64, 128]), new,
                      new + int(math.exp(rng.uniform(0, 12))), rng.choice([-1, 0, 1 << 16, 1 << 20, 1 << 26])))
    refused = plan([("large", c[1], c[2], c[3], c[4]) for c in calls])
    calls = [c for c, (r,) in zip(calls, refused) if not r]
    for call, (rows, slots, shares, parts, size, ws, tiles) in zip(calls, plan(calls)):
        _, tokens, seqs, hq, hkv, dim, new, length, most = call
        assert rows in (16, 32, 256) and slots * rows >= tokens * hq // hkv
        assert most < 0 or ws <= most
        assert (ws == 0) == (parts == 1 and shares == 0)
        if rows < 256:
            assert parts == 1 and shares * hkv <= 512 and shares != 1
            assert ws == 0 or ws >= slots * hkv * 16 + 2 * shares * hkv * rows * (dim + 2) * 4
        else:
            assert -(-tokens * hq // hkv // rows) <= tiles <= slots
            assert shares == 0 and 1 <= parts <= 256 and size >= 16 and slots * hkv * parts * 512 < 2 ** 32
            steps = rng.randint(0, 4000)              # whatever the lengths in device memory are
            each, = plan([("part", steps, size, parts)])[0]
            assert each * parts >= steps and each >= size


def test_tiles_of_any_lengths_fit_the_launch(plan):
    for lengths in _batches(200):
        if sum(lengths):
            (_, _, _, _, _, _, tiles), = plan([("plan", sum(lengths), len(lengths), 8, 2, 128, 9000, 9000, -1)])
            assert tiles >= sum(-(-4 * n // 256) for n in lengths)
    for n in (64, 128, 512, 8192):
        assert plan([("plan", n, 1, 8, 2, 128, 9000, 9000, -1)])[0][6] == n * 4 // 256       # one sequence: no surplus


@pytest.mark.parametrize("most", [2, 64, 102, 512])
def test_shares_hold_every_step_once(plan, most):
    """Share i ends where share i + 1 begins, all have nearly the same number of steps, and a step's share is the one that has it."""
    rng = random.Random(most)
    for total in [1, 7, 8, 15, 16, 17, 100, 4095, 4096, 4097, 123457] + [rng.randint(1, 10 ** 6) for _ in range(10)]:
        n, = plan([("shares", most, total)])[0]
        assert 1 <= n <= most and (n == 1 or total // n >= 8)
        ends = [v for v, in plan([("share", i, n, total) for i in range(n + 1)])]
        assert ends[0] == 0 and ends[-1] == total
        sizes = [b - a for a, b in zip(ends, ends[1:])]
        assert max(sizes) - min(sizes) <= 1 and min(sizes) >= 1
        some = sorted({0, total - 1, *(e for e in ends[:-1]), *(e - 1 for e in ends[1:]), *(rng.randrange(total) for _ in range(20))})
        for x, (i,) in zip(some, plan([("of", x, n, total) for x in some])):
            assert ends[i] <= x < ends[i + 1]


def test_sizes_that_leave_no_grid_are_told(plan):
    assert plan([("large", 122880, 4, 40, 8), ("large", 1 << 22, 1, 32, 8), ("large", 64, 1 << 20, 32, 8), ("large", 1 << 40, 1, 32, 8)]) == [
        (0,), (1,), (1,), (1,)]


# ---- refusals: nothing of these reaches a device ----

def _call(op, **change):
    from paper_2602_16603_amd import binding as B
    c = dict(k_pool=256, v_pool=256, k_scale=256, v_scale=256, num_blocks=8, n_kv_heads=2, head_dim=128)
    b = dict(n_seqs=2, max_blocks=4, cu_seqlens=256, cached_lens=256, block_tables=256)
    a = dict(qkv=256, qkv_stride=1536, n_tokens=2, n_q_heads=8, rope_cos=256, rope_sin=256, max_position=64, q_out=512, q_stride=1024,
             q=256, o=512, o_stride=1024, scale=0.1, max_new=1, max_len=64, workspace=0, workspace_bytes=0, table=256, length=20,
             k_out=256, v_out=256)
    for name, value in change.items():
        (c if name in c else b if name in b else a)[name] = value
    cache, batch = B.fp_kv8_cache(*c.values()), B.fp_kv8_batch(*b.values())
    if op == "append":
        B.fp_op_kv8_append(cache, batch, a["qkv"], a["qkv_stride"], a["n_tokens"], a["n_q_heads"], a["rope_cos"], a["rope_sin"],
                           a["max_position"], a["q_out"], a["q_stride"])
    elif op == "attention":
        B.fp_op_kv8_attention(cache, batch, a["q"], a["q_stride"], a["o"], a["o_stride"], a["n_tokens"], a["n_q_heads"], a["scale"],
                              a["max_new"], a["max_len"], a["workspace"], a["workspace_bytes"])
    else:
        B.fp_op_kv8_gather(cache, a["table"], a["length"], a["k_out"], a["v_out"])


CACHE = [dict(k_pool=0), dict(v_pool=264), dict(k_scale=0), dict(v_scale=258), dict(num_blocks=0), dict(num_blocks=1 << 31), dict(n_kv_heads=0),
         dict(head_dim=96), dict(head_dim=256)]
BATCH = [dict(n_seqs=-1), dict(max_blocks=0), dict(max_blocks=(1 << 26) + 1), dict(cu_seqlens=0), dict(cached_lens=257), dict(block_tables=0)]
APPEND = [dict(n_q_heads=0), dict(n_q_heads=7), dict(n_tokens=-1), dict(n_tokens=1 << 40), dict(max_position=0), dict(qkv=0), dict(qkv=264),
          dict(q_out=0), dict(rope_cos=0), dict(rope_sin=260), dict(qkv_stride=1528), dict(qkv_stride=1540), dict(q_stride=1016),
          dict(q_out=256, q_stride=1024)]
ATTENTION = [dict(n_q_heads=3), dict(n_tokens=-1), dict(n_tokens=1 << 40), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
             dict(scale=math.nan), dict(max_new=0), dict(max_len=0), dict(workspace_bytes=-1), dict(workspace_bytes=256),
             dict(workspace=128, workspace_bytes=256), dict(q=0), dict(o=520), dict(q_stride=1016), dict(o_stride=1028)]
GATHER = [dict(table=0), dict(length=-1), dict(length=1 << 40), dict(k_out=0), dict(v_out=264)]


@pytest.mark.parametrize("op,change", [(op, ch) for op, some in (("append", CACHE + BATCH + APPEND), ("attention", CACHE + BATCH + ATTENTION),
                                                                 ("gather", CACHE + GATHER)) for ch in some], ids=str)
def test_refused(op, change):
    from paper_2602_16603_amd import binding as B
    with pytest.raises(B.FlowPrefillError) as e:
        _call(op, **change)
    assert e.value.status == B.FP_ERR_INVALID and "kv8" in str(e.value)


def test_empty_calls_launch_nothing():
    for change in (dict(n_tokens=0), dict(n_seqs=0)):
        _call("append", **change)
        _call("attention", **change)
    _call("gather", length=0)


def test_workspace_of_a_call_that_would_be_refused_is_nothing():
    from paper_2602_16603_amd import binding as B
    good = (64, 64, 32, 8, 128, 1, 16384)
    assert B.fp_op_kv8_attention_workspace_bytes(*good) > 0
    for i, bad in ((0, 0), (0, 1 << 40), (1, 0), (2, 31), (3, 0), (4, 96), (5, 0), (6, 0)):
        assert B.fp_op_kv8_attention_workspace_bytes(*good[:i], bad, *good[i + 1:]) == 0


def test_models_that_cannot_hold_their_cache_in_8_bits():
    from paper_2602_16603_amd import binding as B
    layer = [dict(attn_norm=16, w_qkv=16, w_o=16, mlp_norm=16, w_gate_up=16, w_down=16)]
    for dtype, kv in ((0, 1), (1, 2), (1, -1)):
        shape = B.fp_shape(1, 64, 2, 2, 64, 64, 1e-5, 1e4, dtype, 16, 4, 16, 0, 0, kv)
        with pytest.raises(B.FlowPrefillError) as e:
            B.fp_model_create(shape, layer)
        assert e.value.status == B.FP_ERR_INVALID and ("8-bit" in str(e.value) or "kv_dtype" in str(e.value))
