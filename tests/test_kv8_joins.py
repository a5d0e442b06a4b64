"""That the calls of kv8_cases.JOINS are cut as they say, without a GPU."""
import pytest

from tests.kv8_cases import JOINS
from tests.test_kv8_plan import plan  # noqa: F401  (a fixture)


@pytest.mark.parametrize("hq,hkv,dim,new,cached,least,alone", JOINS)
def test_parts_of_the_longest_slot(plan, hq, hkv, dim, new, cached, least, alone):
    group, tokens = hq // hkv, sum(new)
    lens = [c + n for c, n in zip(cached, new)]
    (rows, slots, shares, parts, size, ws, tiles), = plan([("plan", tokens, len(new), hq, hkv, dim, max(new), max(lens), -1)])
    steps = -(-max(lens) // 64)
    if rows < 256:
        total = sum(-(-n * group // rows) * max(-(-length // 64), 1) for n, length in zip(new, lens))
        used, = plan([("shares", shares, total)])[0]
        assert steps * used // total >= least                # (nearly as many steps to every share)
        most = shares > 8 * slots
    else:
        each, = plan([("part", steps, size, parts)])[0]
        assert -(-steps // each) >= least
        most = parts > 8
    assert (tokens * hq <= 512 and most) == alone
