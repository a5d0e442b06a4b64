"""How the operators of latent attention cut their work (csrc/latent_plan.h, built for the CPU), without a GPU."""
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
    exe = str(tmp_path_factory.mktemp("latent") / "dump")
    subprocess.run([cxx, "-std=c++17", "-O2", os.path.join(ROOT, "tests", "host", "latent_plan_dump.cpp"), "-o", exe], check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, l)) for l in lines) + "\n", stdout=subprocess.PIPE, text=True,
                             check=True, timeout=300).stdout
        return [tuple(map(int, l.split())) for l in out.splitlines()]
    return run


def _calls(count):
    rng = random.Random(5)
    for _ in range(count):
        seqs = rng.choice([1, 1, 2, 7, 64, 500])
        new = rng.choice([1, 1, 1, 2, 5, 40, 512, 4000])
        tokens = rng.randint(1, seqs * new)
        heads = rng.choice([1, 4, 16, 20, 33, 64, 65, 128, 130, 1000])
        yield tokens, seqs, heads, new, rng.choice([1, 16, 100, 250, 2000, 30000, 10 ** 6, 2 ** 30])


def test_head_tiles_have_all_heads(plan):
    heads = list(range(1, 700)) + [4096, 65536]
    for h, (tiles, group, *_rest) in zip(heads, plan([("plan", 1, 1, h, 512, 10, 1, 100, -1) for h in heads])):
        assert 1 <= group <= 64 and tiles * group >= h > (tiles - 1) * group


def test_tiles_bound_what_any_split_of_the_tokens_needs(plan):
    rng = random.Random(6)
    for _ in range(300):
        new = [rng.choice([0, 1, 1, 2, 63, 64, 65, 300]) for _ in range(rng.randint(1, 30))]
        heads, tokens = rng.choice([1, 4, 20, 33, 64, 130]), sum(new)
        if tokens == 0:
            continue
        (tiles, group, rows, slots, bound, *_), (_, e_bound, *_) = plan([("plan", tokens, len(new), heads, 512, 10, max(new), 64, 0),
                                                                       ("expanded", tokens, len(new), heads, 128, max(new), 64, 0)])
        assert sum(-(-n * group // rows) for n in new) <= bound <= slots
        assert sum(-(-n // 256) for n in new) <= e_bound


def test_shares_stay_within_the_workspace(plan):
    rng = random.Random(7)
    calls, given = [], []
    for tokens, seqs, heads, new, length in _calls(2000):
        for ws in (-1, 0, rng.randint(0, 1 << 26)):
            calls.append(("plan", tokens, seqs, heads, rng.choice([128, 256, 512]), rng.choice([1, 100, 1 << 26]), new, length, ws))
            given.append(ws)
    for call, ws, (head_tiles, _, rows, slots, tiles, shares, workspace, slab) in zip(calls, given, plan(calls)):
        assert rows in (32, 64)
        if shares == 0:
            assert workspace == 0
            continue
        assert 2 <= shares <= 256 and shares * head_tiles <= 256 + head_tiles
        assert workspace == -(-slots * 16 // 256) * 256 + 2 * shares * head_tiles * slab
        assert ws < 0 or workspace <= ws
        # Steps of all slots are counted in 32 bits.
        assert slots * ((call[5] + 1) // 2 + 1) < 2 ** 31


def test_a_smaller_workspace_never_gives_more_shares(plan):
    for tokens, seqs, heads, new, length in _calls(200):
        sizes = [0, 1 << 16, 1 << 20, 1 << 22, 1 << 24, 1 << 26, -1]
        shares = [p[5] for p in plan([("plan", tokens, seqs, heads, 512, 1000, new, length, s) for s in sizes])]
        most = shares[-1]
        assert all(s <= most for s in shares if most)


def test_expanded_parts_stay_within_the_workspace(plan):
    rng = random.Random(8)
    calls = [("expanded", t, s, h, rng.choice([64, 128]), n, length, rng.choice([-1, 0, rng.randint(0, 1 << 26)])) for t, s, h, n, length in _calls(2000)]
    for (_, tokens, seqs, heads, v, _, length, ws), (slots, tiles, parts, steps, workspace) in zip(calls, plan(calls)):
        assert 1 <= parts <= 256 and tiles * heads * parts * 512 < 2 ** 32
        assert workspace == (slots * heads * parts * 256 * (v + 2) * 4 if parts > 1 else 0)
        assert ws < 0 or workspace <= ws
        if parts > 1:
            assert parts * steps >= -(-length // 64) or parts < -(-length // 64)


def test_launches_that_are_taken_have_fewer_threads_than_a_grid_may(plan):
    rng = random.Random(9)
    for _ in range(3000):
        tokens, seqs, heads = (int(2 ** rng.uniform(0, 25)) for _ in range(3))
        heads = min(heads, 65536)
        (large,), (head_tiles, _, rows, slots, tiles, *_), (e_slots, e_tiles, parts, *_) = plan([
            ("large", tokens, seqs, heads), ("plan", tokens, seqs, heads, 512, 1 << 26, 1, 64, 0), ("expanded", tokens, seqs, heads, 128, 1, 64, 0)])
        if large:
            continue
        assert (tiles + 7) // 8 * 8 * head_tiles * rows * 8 < 2 ** 32
        assert e_tiles * heads * parts * 512 < 2 ** 32
        assert (tokens * (1 + -(-heads // 32)) + 3) // 4 * 256 < 2 ** 32
        assert slots < 2 ** 31 and e_slots < 2 ** 31


def test_one_slot_is_cut_into_no_more_parts_than_the_bound(plan):
    """One token of up to 64 heads is one slot, whatever the bound of slots with its gaps says (twice as many where its heads fill one):
    128 shares, or as many as have 16 steps of 32 keys each."""
    calls = [("plan", 1, 1, h, latent, 1 << 16, 1, length, ws) for h in range(1, 65) for latent in (128, 256, 512)
             for length in (600, 8000, 32768, 65536, 100000, 1 << 20) for ws in (-1, 1 << 27)]
    for call, (head_tiles, _, _, _, tiles, shares, *_) in zip(calls, plan(calls)):
        assert head_tiles == tiles == 1
        assert shares == min(max(128, -(-call[7] // 32) // 16), 256), call
    # ... nor are more of them ever in use than there is work for.
    totals = [1, 2, 3, 4, 5, 7, 8, 9, 127, 511, 512, 513, 1025, 2 ** 31 - 1]
    for most in (1, 2, 128, 256):
        for total, (used,) in zip(totals, plan([("shares", most, t) for t in totals])):
            assert used == min(max(total // 4, 1), most)


def test_products_per_head_have_a_workgroup_for_every_cu_where_there_are_rounds_enough(plan):
    """A workgroup's run of tokens is a round of 128, or so many that a shorter one would give more workgroups than CUs; runs are not
    so short that there are more than a workgroup for every CU."""
    rng = random.Random(10)
    calls = [("heads", m, h, n, k) for h in (4, 20, 32, 40, 128) for m in (300, 700, 2000, 4096) for n, k in ((512, 128), (128, 512), (256, 64))]
    calls += [("heads", int(2 ** rng.uniform(0, 15)), rng.randint(1, 300), 8 * rng.randint(1, 200), rng.choice([64, 128, 256, 512])) for _ in range(2000)]
    for (_, m, heads, n, k), (_, run, tiles) in zip(calls, plan(calls)):
        assert tiles == -(-n // (512 if k == 64 else 65536 // k)) and 65536 // k * k * 2 <= 128 << 10
        assert run % 128 == 0 and run > 0
        assert run == 128 or heads * tiles * -(-m // (run - 128)) > 256, (m, heads, n, k, run)
        assert heads * tiles * -(-m // run) <= max(256, heads * tiles)
    for m, heads, wide in ((64, 128, 0), (65, 128, 1), (256, 32, 0), (257, 32, 1), (384, 20, 0), (385, 20, 1), (32, 1000, 0), (33, 1000, 1), (2, 65536, 0)):
        assert plan([("heads", m, heads, 128, 512)])[0][0] == wide
    for k in (8, 32, 96, 120, 192, 384, 1024):
        assert plan([("heads", 1 << 20, 128, 128, k)])[0][0] == 0
