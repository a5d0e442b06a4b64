"""The 8-bit cache's operators at the limits of what their calls allow, against the definition in 64 bits."""
import pytest
import torch

from tests import kv8_util as U
from tests.kv8_cases import JOINS
from tests.test_gpu_kv8 import _attention_case, _binding, _normal

pytestmark = pytest.mark.gpu


def _spiked(batch, q, hq, dim, exponent, seed):
    """Rows of q replaced, two in three of every head: one channel alone, of size 2^exponent, either sign."""
    g = torch.Generator().manual_seed(seed)
    rows = q.view(-1, hq, dim).clone()
    spiked = torch.arange(rows.shape[0] * hq).reshape(rows.shape[0], hq) % 3 > 0
    value = (1 + torch.rand(spiked.shape, generator=g)) * 2.0 ** exponent * torch.where(torch.rand(spiked.shape, generator=g) < 0.5, -1.0, 1.0)
    rows[spiked] = 0
    rows[..., 0][spiked] = value[spiked].bfloat16()
    return rows.reshape(q.shape), spiked


@pytest.mark.parametrize("exponent", [24, 31, 40, 100])
@pytest.mark.parametrize("hq,hkv,dim,new,cached", [(4, 2, 64, [1], [40]), (4, 1, 128, [1, 2], [1300, 30]), (8, 1, 64, [5], [1000]), (8, 1, 128, [5], [90]),
                                                   (8, 2, 64, [150, 1], [0, 500]), (8, 1, 128, [70], [2500])])
def test_attention_of_scores_that_fp32_spaces_wide(hq, hkv, dim, new, cached, exponent):
    """Finite scores of which one takes all: a score next to the largest lies 2^exponent * 2^-9 * scale > 2^10 below it, so its weight is
    zero, and rows that see several keys of the largest score get their values' mean.  Weights are one, their sum is a count: what is
    left are the sum over the values and the division in fp32, and the output's rounding.  Ordinary rows lie between those rows."""
    B = _binding()
    cache, batch, q = _attention_case(hq, hkv, dim, new, cached, 500 + exponent, garbage=True)
    q, spiked = _spiked(batch, q, hq, dim, exponent, 1)
    for name in "kv":
        cache.scale[name].fill_(1.0)
    scale = dim ** -0.5
    ref, tol = cache.attention(q, hq, batch.cu, batch.cached, batch.table, scale)
    keys = max(c + n for c, n in zip(cached, new))
    exact = (U.HALF_BF16 * (1 + 4 * U.HALF_FP32) + 4 * U.HALF_FP32) * ref.abs() + (keys + 4) * U.HALF_FP32 * U.TOP
    one = spiked.repeat_interleave(dim, 1)
    ordinary = torch.where(spiked[..., None], 0.0, q.view(-1, hq, dim).double()).reshape(q.shape).bfloat16()
    tol = torch.where(one, exact, cache.attention(ordinary, hq, batch.cu, batch.cached, batch.table, scale)[1])
    assert not ref.isnan().any()
    for workspace in (True, 0):
        U.check(U.attend(B, cache, cache.upload(), batch, q.cuda(), hq, scale, workspace=workspace), ref, tol, workspace)


def test_a_task_with_a_table_that_positions_in_32_bits_cannot_span_is_refused():
    """As the single operators refuse it: from 2^27 entries a row on, 16 times their number leaves 32 bits and every sequence looked idle."""
    import numpy as np
    from paper_2602_16603_amd import inputs as I
    B = _binding()
    from tests.test_gpu_kv8_model import _model
    model, _ = _model(I.TINY.with_layers(1), 3, 8, 64)
    hidden = I.make_hidden(20, I.TINY.hidden, 3, torch.bfloat16, "cuda")
    with pytest.raises(B.FlowPrefillError) as e:
        model.begin(hidden, [20], [0], np.zeros((1, (1 << 26) + 1), dtype=np.int32))
    assert e.value.status == B.FP_ERR_INVALID and "max_blocks" in str(e.value)
    task = model.begin(hidden, [20], [0], np.array([[5, 2, -1]], dtype=np.int32))
    task.run_to_completion()
    assert task.hidden().isfinite().all()
    task.end()
    model.close()


@pytest.mark.parametrize("evicted", [(), ((100, 300),), ((0, 70), (90, 92), (400, 480))], ids=["whole", "a part", "several"])
@pytest.mark.parametrize("hq,hkv,dim,new,cached,least,alone", JOINS)
def test_attention_joined_over_many_parts(hq, hkv, dim, new, cached, least, alone, evicted):
    """Up to 137 partial results of a row (test_kv8_joins.py), with parts that saw no key among them, and the same bits every time."""
    B = _binding()
    print("join", hq, hkv, dim, sum(new), max(cached), evicted, flush=True)
    cache, batch, q = _attention_case(hq, hkv, dim, new, cached, 700, garbage=True)
    long = cached.index(max(cached))
    for lo, hi in evicted:
        batch.table[long][lo:hi] = [-1] * (hi - lo)
    ref, tol = cache.attention(q, hq, batch.cu, batch.cached, batch.table, dim ** -0.5)
    dev, qd = cache.upload(), q.cuda()
    first = U.attend(B, cache, dev, batch, qd, hq, dim ** -0.5)
    U.check(first, ref, tol)
    for _ in range(3):
        assert torch.equal(U.attend(B, cache, dev, batch, qd, hq, dim ** -0.5), first)
    full = B.fp_op_kv8_attention_workspace_bytes(q.shape[0], len(new), hq, hkv, dim, batch.max_new, batch.max_len)
    for workspace in (full // 3, 0):
        U.check(U.attend(B, cache, dev, batch, qd, hq, dim ** -0.5, workspace=workspace), ref, tol, workspace)
