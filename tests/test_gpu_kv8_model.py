"""Models whose KV cache is held in 8 bits: the prefill path with the 8-bit cache's operators as its operators 2 and 3."""
import numpy as np
import pytest
import torch

from oracle import prefill_oracle as O
from paper_2602_16603_amd import inputs as I
from tests import kv8_util as U
from tests.util import TOL, fro_rel_err, max_rel_err, oracle_layers, oracle_shape

pytestmark = pytest.mark.gpu

WIDE = I.ShapeSpec(2, 256, 8, 2, 128, 512, 1e-5, 10000.0)


def _model(spec, seed, blocks, max_position, kv=1):
    from paper_2602_16603_amd import runner
    weights = I.make_weights(spec, seed, torch.bfloat16, "cpu")
    I.randomize_gains(weights, seed)
    return runner.PrefillModel(spec, weights, 1, blocks, max_position, kv_dtype=kv), weights


def _layer_over_held(spec, w, x, lengths, cached, held):
    """One layer in 64 bits whose attention reads the keys and values that the cache holds."""
    sh = oracle_shape(spec)
    x = x.double()
    qkv = O.linear(O.rmsnorm(x, w.attn_norm, spec.rms_eps), w.w_qkv)
    out, lo = [], 0
    for n, c, (k, v) in zip(lengths, cached, held):
        pos = torch.arange(c, c + n)
        q = O.rope_rotate(qkv[lo:lo + n, :sh.q_width].reshape(n, spec.n_q_heads, spec.head_dim), pos, spec.rope_theta)
        out.append(O.causal_attention(q, k.cpu(), v.cpu(), pos).reshape(n, sh.q_width))
        lo += n
    x = x + O.linear(torch.cat(out), w.w_o)
    h = O.rmsnorm(x, w.mlp_norm, spec.rms_eps)
    return x + O.linear(O.silu_mul(O.linear(h, w.w_gate_up)), w.w_down), qkv


@pytest.mark.parametrize("spec", [I.TINY.with_layers(1), WIDE.with_layers(1)], ids=["64", "128"])
@pytest.mark.parametrize("lengths", [[256], [1, 300, 17, 0, 130], [3], [1, 1, 1]])
def test_layer_matches_the_oracle_over_what_the_cache_holds(spec, lengths):
    total = sum(lengths)
    model, weights = _model(spec, 5, 256, 1024)
    hidden = I.make_hidden(total, spec.hidden, 5, torch.bfloat16, "cpu")
    table, _ = I.permuted_block_tables(lengths, None, 16, 256, seed=3)
    task = model.begin(hidden.cuda(), lengths, [0] * len(lengths), table)
    task.run_to_completion()
    held = [task.kv(0, s) for s in range(len(lengths))]
    w = oracle_layers(weights)[0]
    ref, qkv = _layer_over_held(spec, w, hidden, lengths, [0] * len(lengths), held)
    assert max_rel_err(task.hidden(), ref) <= TOL["bf16"]
    # What is held: half an e4m3 step from the oracle's, which the projection's own tolerance moves.
    lo, hq, hkv, dim = 0, spec.n_q_heads, spec.n_kv_heads, spec.head_dim
    for n, (k, v) in zip(lengths, held):
        rows = qkv[lo:lo + n].reshape(n, hq + 2 * hkv, dim)
        for got, want in ((k, O.rope_rotate(rows[:, hq:hq + hkv], torch.arange(n), spec.rope_theta)), (v, rows[:, hq + hkv:])):
            if n:
                slack = TOL["bf16"] * want.abs().max()
                assert ((got.cpu().double() - want).abs() <= 2.0 ** -4 * (want.abs() + slack) + slack).all()
        lo += n
    task.end()
    model.close()


def test_stack_stays_near_the_oracle():
    """Two layers against the oracle without any rounding: keys and values carry half an e4m3 step, 2^-4, of which a softmax average
    over n keys leaves less; the residual stream that the attention adds to is of size one, its addition about a tenth of that."""
    spec, lengths = I.TINY, [200, 60]
    model, weights = _model(spec, 6, 64, 256)
    hidden = I.make_hidden(260, spec.hidden, 6, torch.bfloat16, "cpu")
    task = model.begin(hidden.cuda(), lengths)
    task.run_to_completion()
    ref, _ = O.prefill(oracle_shape(spec), oracle_layers(weights), hidden, I.cu_seqlens_of(lengths))
    assert fro_rel_err(task.hidden(), ref) <= 2.0 ** -4
    task.end()
    model.close()


def test_parked_and_resumed_at_every_boundary_gives_the_same_bits():
    from paper_2602_16603_amd import binding as B
    spec, lengths = WIDE, [100, 41]
    model, _ = _model(spec, 7, 64, 256)
    hidden = I.make_hidden(141, spec.hidden, 7, torch.bfloat16, "cuda")
    other = I.make_hidden(30, spec.hidden, 8, torch.bfloat16, "cuda")
    whole = model.begin(hidden, lengths)
    whole.run_to_completion()
    want = [whole.hidden()] + [t for layer in range(2) for s in range(2) for t in whole.kv(layer, s)]
    task = model.begin(hidden, lengths)
    while True:
        st, _ = task.advance(1)
        if st == B.FP_DONE:
            break
        assert task.preempt() == B.FP_PREEMPTED
        short = model.begin(other, [30])
        short.run_to_completion()
        short.end()
        task.resume()
    got = [task.hidden()] + [t for layer in range(2) for s in range(2) for t in task.kv(layer, s)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    task.end()
    whole.end()
    model.close()


@pytest.mark.parametrize("chunks", [[48, 96, 16, 40], [33, 100, 1, 1, 1, 64]])
def test_chunks_and_single_tokens_continue_the_cache(chunks):
    """A prompt in chunks, single tokens among them: the first layer's cache is that of the whole prompt (blocks that were completed by
    several chunks have been rounded again, by half a step of the subnormal codes at most), the output that of the oracle over
    what is held."""
    spec = WIDE.with_layers(1)
    total = sum(chunks)
    model, weights = _model(spec, 9, 64, 256)
    hidden = I.make_hidden(total, spec.hidden, 9, torch.bfloat16, "cuda")
    table = np.random.RandomState(0).permutation(64)[:16].astype(np.int32).reshape(1, 16)
    whole = model.begin(hidden, [total], [0], table)
    whole.run_to_completion()
    k0, v0 = (t.clone() for t in whole.kv(0, 0))
    whole.end()
    w = oracle_layers(weights)[0]
    at = 0
    for n in chunks:
        task = model.begin(hidden[at:at + n].contiguous(), [n], [at], table)
        task.run_to_completion()
        held = [task.kv(0, 0)]
        ref, _ = _layer_over_held(spec, w, hidden[at:at + n].cpu(), [n], [at], held)
        assert max_rel_err(task.hidden(), ref) <= TOL["bf16"], at
        at += n
        task.end()
    for got, want in zip(held[0], (k0, v0)):
        # The projection of another number of rows adds up in another order, so a value next to a border may move by a step.
        step = torch.maximum(want.float().abs() * 2.0 ** -3, want.float().abs().max() * 2.0 ** -16)
        assert ((got.float() - want.float()).abs() <= 1.01 * step + TOL["bf16"] * 2.0 ** -4).all()
    model.close()


def test_mixture_of_experts_model():
    spec = I.TINY_MOE
    model, weights = _model(spec, 10, 64, 512)
    plain, _ = _model(spec, 10, 64, 512, kv=0)
    hidden = I.make_hidden(150, spec.hidden, 10, torch.bfloat16, "cuda")
    outs = []
    for m in (model, plain):
        task = m.begin(hidden, [90, 60])
        task.run_to_completion()
        outs.append(task.hidden())
        task.end()
    assert fro_rel_err(outs[0], outs[1]) <= 2.0 ** -4
    model.close()
    plain.close()


def test_pools_scales_and_tables_are_what_the_operators_take():
    """The single operators on a model's own pools: gathering a layer by hand, and a decode step's attention over it."""
    from paper_2602_16603_amd import binding as B
    from paper_2602_16603_amd.runner import copy_from_device_ptr
    spec, lengths = WIDE, [77, 30]
    hq, hkv, dim, blocks = spec.n_q_heads, spec.n_kv_heads, spec.head_dim, 32
    model, _ = _model(spec, 11, blocks, 256)
    hidden = I.make_hidden(107, spec.hidden, 11, torch.bfloat16, "cuda")
    task = model.begin(hidden, lengths)
    task.run_to_completion()
    ks, vs = B.fp_model_kv_scales(model.handle)
    cos, sin = B.fp_model_rope_tables(model.handle)
    assert torch.equal(copy_from_device_ptr(cos, (256, dim // 2), torch.float32).cpu(), U.rope_tables(256, dim, spec.rope_theta)[0])
    table = torch.tensor(task.block_tables(), dtype=torch.int32, device="cuda")
    for layer in range(2):
        k_pool, v_pool, _ = task.kv_pools(layer)
        at = layer * blocks * hkv * 4
        cache = B.fp_kv8_cache(k_pool, v_pool, ks + at, vs + at, blocks, hkv, dim)
        for s, n in enumerate(lengths):
            k = torch.empty((n, hkv, dim), dtype=torch.bfloat16, device="cuda")
            v = torch.empty_like(k)
            B.fp_op_kv8_gather(cache, table[s].data_ptr(), n, k.data_ptr(), v.data_ptr())
            torch.cuda.synchronize()
            k2, v2 = task.kv(layer, s)
            assert torch.equal(k, k2) and torch.equal(v, v2)
            assert k.abs().max() > 0 and v.abs().max() > 0
        # one query per sequence over it (the last position's)
        q = I.normal_tensor((2, hq * dim), 1.0, 12 + layer, torch.bfloat16, "cuda")
        cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        cached = torch.tensor([n - 1 for n in lengths], dtype=torch.int32, device="cuda")
        batch = B.fp_kv8_batch(2, table.shape[1], cu.data_ptr(), cached.data_ptr(), table.data_ptr())
        o = torch.empty_like(q)
        B.fp_op_kv8_attention(cache, batch, q.data_ptr(), hq * dim, o.data_ptr(), hq * dim, 2, hq, dim ** -0.5, 1, 77)
        torch.cuda.synchronize()
        for s, n in enumerate(lengths):
            k, v = task.kv(layer, s)
            ref = O.causal_attention(q[s:s + 1].cpu().view(1, hq, dim), k.cpu(), v.cpu(), torch.tensor([n - 1])).reshape(1, -1)
            assert max_rel_err(o[s:s + 1], ref) <= 3 * U.HALF_BF16          # probabilities, their sum, the output
    task.end()
    model.close()
