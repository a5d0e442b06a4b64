"""Models with an 8-bit cache whose sequences are long enough for the attention to be cut over its keys: its partial results lie in the
task's workspace, in the region that the projections' partial sums use before and after it."""
import numpy as np
import pytest
import torch

from paper_2602_16603_amd import inputs as I
from tests.test_gpu_kv8_model import WIDE, _layer_over_held, _model
from tests.util import TOL, max_rel_err, oracle_layers

pytestmark = pytest.mark.gpu

NARROW = I.TINY                                       # heads of 64


def _is_cut(spec, new, cached):
    from paper_2602_16603_amd import binding as B
    return B.fp_op_kv8_attention_workspace_bytes(sum(new), len(new), spec.n_q_heads, spec.n_kv_heads, spec.head_dim, max(new),
                                                 max(n + c for n, c in zip(new, cached))) > 0


def _table(rows, width, blocks, seed=0):
    return np.random.RandomState(seed).permutation(blocks)[:rows * width].astype(np.int32).reshape(rows, width)


@pytest.mark.parametrize("spec", [WIDE.with_layers(1), NARROW.with_layers(1)], ids=["128", "64"])
@pytest.mark.parametrize("tasks", [[[1500], [3], [100], [1], [64], [256]], [[1310, 900], [100, 2], [1, 1], [5, 70], [0, 130], [40, 0]]],
                         ids=["one", "packed"])
def test_layers_match_the_oracle_where_the_attention_is_cut(spec, tasks):
    """Chunks, single tokens and both in one task, each against the oracle over the keys and values that the cache then holds."""
    seqs = len(tasks[0])
    model, weights = _model(spec, 21, 2 * 128, 2048)
    table = _table(seqs, 128, 256)
    w = oracle_layers(weights)[0]
    cached, cut = [0] * seqs, 0
    for i, new in enumerate(tasks):
        hidden = I.make_hidden(sum(new), spec.hidden, 30 + i, torch.bfloat16, "cuda")
        cut += _is_cut(spec, new, cached)
        task = model.begin(hidden, new, cached, table)
        task.run_to_completion()
        held = [task.kv(0, s) for s in range(seqs)]
        ref, _ = _layer_over_held(spec, w, hidden.cpu(), new, cached, held)
        assert max_rel_err(task.hidden(), ref) <= TOL["bf16"], (i, new)
        task.end()
        cached = [a + b for a, b in zip(cached, new)]
    assert cut >= len(tasks) - 1                      # (all but the prompts themselves)
    model.close()


@pytest.mark.parametrize("chunk", [[1], [60], [100], [100, 1]])
def test_parked_behind_a_cut_attention_keeps_its_bits(chunk):
    """Parked at every boundary, between the cut attention and the projection that takes its region over among them, while another
    task with a cut attention of its own runs to its end."""
    from paper_2602_16603_amd import binding as B
    spec, before, seqs = WIDE, 1296, len(chunk)       # (a whole number of blocks: a task that runs again finds the same cache)
    model, _ = _model(spec, 22, 3 * 96, 1536)
    table = _table(3, 96, 288, 1)
    mine, others = table[:seqs], table[2:]
    for rows, n in ((mine, seqs), (others, 1)):
        task = model.begin(I.make_hidden(before * n, spec.hidden, 40, torch.bfloat16, "cuda"), [before] * n, [0] * n, rows)
        task.run_to_completion()
        task.end()
    hidden = I.make_hidden(sum(chunk), spec.hidden, 41, torch.bfloat16, "cuda")
    other = I.make_hidden(2, spec.hidden, 42, torch.bfloat16, "cuda")
    cached = [before] * seqs
    assert _is_cut(spec, chunk, cached) and _is_cut(spec, [2], [before])

    def results(task):
        return [task.hidden().clone()] + [t.clone() for layer in range(2) for s in range(seqs) for t in task.kv(layer, s)]
    task = model.begin(hidden, chunk, cached, mine)
    task.run_to_completion()
    want = results(task)
    task.end()
    task = model.begin(hidden, chunk, cached, mine)
    parked = 0
    while True:
        st, _ = task.advance(1)
        if st == B.FP_DONE:
            break
        assert task.preempt() == B.FP_PREEMPTED
        parked += 1
        between = model.begin(other, [2], [before], others)
        between.run_to_completion()
        between.end()
        task.resume()
    assert parked == 17 and all(torch.equal(a, b) for a, b in zip(results(task), want))
    task.end()
    model.close()
