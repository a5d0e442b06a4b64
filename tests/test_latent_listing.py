"""The assembly that latent attention's kernels compile to, without a GPU.

Their sums are matrix instructions written in assembly, which the compiler neither sees nor waits for (latent_add_product), and their loads
into LDS set m0 themselves (latent_load_lds).  So the listing of each kernel is walked over all its branches: vector registers that such an
instruction reads were not written by a vector instruction in the two slots before it; what it writes is not touched for 18 slots but by another
matrix instruction that accumulates into just these registers; and nothing of the compiler's reads the m0 that a load has left."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_16603_amd.csrc import build

FRESH, LATE = 2, 18
REG = re.compile(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)")


def _regs(text):
    return {r for a, b, c in REG.findall(text) for r in (range(int(a), int(b) + 1) if a else (int(c),))}


class Line:
    """One instruction: its registers by role, the slots it takes, where it may go."""

    def __init__(self, text, inline):
        self.text, self.inline = text, inline
        self.op = text.split()[0]
        args = [a.strip() for a in re.split(r",(?![^\[]*\])", text[len(self.op):])]
        self.slots = int(args[0], 0) + 1 if self.op == "s_nop" else 1
        self.product = self.op.startswith("v_mfma")
        self.all = set().union(*[_regs(a) for a in args])
        self.into = _regs(args[0])
        self.sources = [_regs(a) for a in args[1:4]] if self.product else []
        vector = self.op.startswith("v_") and not self.product and not re.match(r"v_(cmp|read)", self.op)
        self.writes = (self.all if "swap" in self.op else self.into) if vector else set()
        m0 = [bool(re.search(r"\bm0\b", a)) for a in args]
        self.sets_m0 = m0[0] and not self.op.startswith(("s_cmp", "s_bitcmp"))
        self.reads_m0 = any(m0[0 if not self.sets_m0 else 1:]) or bool(re.search(r"movrel|sendmsg|gws|\blds\b|_lds_", text))
        self.target = args[0] if re.match(r"s_c?branch", self.op) else None
        self.ends = self.op in ("s_branch", "s_endpgm")


def _functions(listing):
    """name -> [Line or label]"""
    out, name, inline = {}, None, False
    for raw in listing.split("\n"):
        text = raw.split(";")[0].strip()
        if "#ASMSTART" in raw or "#ASMEND" in raw:
            inline = "#ASMSTART" in raw
        elif re.match(r"_Z\w+:", text):
            name = text[:-1]
            out[name] = []
        elif text.startswith(".Lfunc_end"):
            name = None
        elif name and re.match(r"\.LBB\w+:", text):
            out[name].append(text[:-1])
        elif name and raw.startswith("\t") and text and text[0] != ".":
            out[name].append(Line(text, inline))
    return out


def _faults(body):
    """What is wrong in one function; a state is (slots since each register was written by a vector instruction, slots since a product in
    assembly wrote it with the registers that it wrote, whether m0 is a load's)."""
    blocks, labels = [[]], {}
    for x in body:
        if isinstance(x, str):
            if blocks[-1]:
                blocks.append([])
            labels[x] = len(blocks) - 1
        else:
            blocks[-1].append(x)
            if x.target or x.ends:
                blocks.append([])
    if not blocks[-1]:
        blocks.pop()
    entry, work, faults = {0: ({}, {}, False)}, [0], set()
    while work:
        at = work.pop()
        fresh, late, m0 = dict(entry[at][0]), dict(entry[at][1]), entry[at][2]
        for x in blocks[at]:
            if x.inline and x.product:
                faults.update(f"{x.text}: v{r} written {d} slots before" for r, d in fresh.items() if any(r in s for s in x.sources))
            if x.product:
                exact = x.into == x.sources[2]
                for r, (_, group) in late.items():
                    if r in x.all and not (exact and group == frozenset(x.into) and not any(r in s for s in x.sources[:2])):
                        faults.add(f"{x.text}: v{r} is on its way")
            else:
                faults.update(f"{x.text}: v{r} is on its way" for r in late if r in x.all)
            if x.reads_m0 and m0 and not x.inline:
                faults.add(f"{x.text}: m0 is a load's")
            if x.sets_m0:
                m0 = x.inline
            fresh = {r: d + x.slots for r, d in fresh.items() if d + x.slots < FRESH}
            late = {r: (d + x.slots, g) for r, (d, g) in late.items() if d + x.slots < LATE}
            fresh.update((r, 0) for r in x.writes)
            if x.inline and x.product:
                late.update((r, (0, frozenset(x.into))) for r in x.into)
        last = blocks[at][-1]
        goes = [labels[last.target]] if last.target else []
        if not last.ends and at + 1 < len(blocks):
            goes.append(at + 1)
        for to in goes:
            if to not in entry:
                entry[to] = (dict(fresh), dict(late), m0)
                work.append(to)
                continue
            f, l, m = entry[to]
            nf = {r: min(f.get(r, FRESH), fresh.get(r, FRESH)) for r in {*f, *fresh}}
            nl = {r: _nearer(l.get(r), late.get(r)) for r in {*l, *late}}
            if (nf, nl, m or m0) != (f, l, m):
                entry[to] = (nf, nl, m or m0)
                work.append(to)
    return faults


def _nearer(a, b):
    if a is None or b is None:
        return a or b
    return min(a[0], b[0]), a[1] if a[1] == b[1] else frozenset()


def _asm(*lines):
    return "\n".join(["\t;;#ASMSTART", *("\t" + x for x in lines), "\t;;#ASMEND"])


PRODUCT = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]"


@pytest.mark.parametrize("body,bad", [
    (["\tds_read_b128 v[8:11], v20", _asm(PRODUCT), _asm(PRODUCT), _asm("s_nop 15", "s_nop 15"), "\tv_add_f32_e32 v5, v0, v1"], False),
    ([_asm(PRODUCT), "\ts_nop 15", "\tv_add_f32_e32 v5, v0, v1"], True),                                  # 17 slots
    ([_asm(PRODUCT), "\ts_nop 3", "\tglobal_store_dwordx4 v[30:31], v[0:3], off"], True),
    ([_asm(PRODUCT), "\tv_mfma_f32_16x16x32_bf16 v[2:5], v[8:11], v[12:15], v[2:5]"], True),                  # overlaps, not the same
    ([_asm(PRODUCT), "\tv_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]"], True),
    (["\tv_mov_b32_e32 v9, 0", "\ts_nop 0", _asm(PRODUCT)], True),
    (["\tv_mov_b32_e32 v9, 0", _asm("s_nop 1", PRODUCT)], False),
    (["\tv_permlane32_swap_b32 v7, v9", _asm(PRODUCT)], True),
    # Round a loop: the sums are touched at its head.
    ([".LBB0_1:", "\tv_mul_f32_e32 v0, v0, v30", "\ts_nop 7", _asm(PRODUCT), "\ts_cbranch_scc1 .LBB0_1", _asm("s_nop 15", "s_nop 15"),
      "\tv_add_f32_e32 v5, v0, v1"], True),
    ([".LBB0_1:", "\ts_nop 15", "\ts_nop 15", "\tv_mul_f32_e32 v0, v0, v30", "\ts_nop 7", _asm(PRODUCT), "\ts_cbranch_scc1 .LBB0_1"], False),
    (["\ts_mov_b32 m0, s3", _asm("s_add_u32 m0, s4, 0", "s_nop 4", "buffer_load_dwordx4 v1, s[0:3], 0 offen lds"), "\tv_movrels_b32 v2, v3 m0"], True),
    ([_asm("s_add_u32 m0, s4, 0"), "\ts_mov_b32 s9, m0"], True),
    ([_asm("s_add_u32 m0, s4, 0"), "\ts_mov_b32 m0, s9", "\ts_mov_b32 s9, m0"], False),
])
def test_the_walk_finds_what_it_is_for(body, bad):
    found = _faults(_functions("\n".join(["_Z1f:", *body, "\ts_endpgm", ".Lfunc_end0:"]))["_Z1f"])
    assert bool(found) == bad, found


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("no hipcc")
    folder, jobs = tmp_path_factory.mktemp("listing"), []
    for name in ("latent_attention", "latent_expanded"):
        out = str(folder / (name + ".s"))
        jobs.append((name, out, subprocess.Popen([hipcc, *build.FLAGS, *build.EXTRA.get(name + ".hip", []), "--cuda-device-only", "-S",
                                                  os.path.join(build.HERE, name + ".hip"), "-o", out], stderr=subprocess.DEVNULL)))
    assert all(job.wait() == 0 for _, _, job in jobs)
    return {name: _functions(open(out).read()) for name, out, _ in jobs}


@pytest.mark.parametrize("name,kernels", [("latent_attention", 12), ("latent_expanded", 8)])
def test_products_in_assembly_keep_their_distances_and_m0_is_the_loads_alone(listings, name, kernels):
    with_products = {k: body for k, body in listings[name].items() if any(isinstance(x, Line) and x.inline and x.product for x in body)}
    assert len(with_products) == kernels                    # (every shape of the attention itself)
    for kernel, body in with_products.items():
        assert any(isinstance(x, Line) and x.inline and x.sets_m0 for x in body), kernel
        assert _faults(body) == set(), kernel


@pytest.mark.parametrize("name", ["latent_attention", "latent_expanded"])
def test_kernels_settle_their_products_before_they_read_the_sums(name):
    """In the file that makes them, not only where the wait is written: behind the last product's place, and at least once more for the sums that
    are rescaled on the way."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.HERE, name + ".hip")).read())
    products = [m.start() for m in re.finditer(r"\blatent_add_product\b", text)]
    settles = [m.start() for m in re.finditer(r"\blatent_settle\(\)", text)]
    assert products and len(settles) >= 2 and settles[-1] > products[-1]


def test_no_other_kernel_makes_products_that_are_not_walked():
    users = {f for f in os.listdir(build.HERE) if f.endswith(".hip") and "latent_add_product" in open(os.path.join(build.HERE, f)).read()}
    assert users == {"latent_attention.hip", "latent_expanded.hip"}
