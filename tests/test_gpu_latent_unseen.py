"""What a row of latent attention does not see has no influence on it: numbers that are not finite in queries, keys and values, beside blocks
that are not there and in every shape and cut of the operators."""
import math

import pytest
import torch

from tests import latent_util as U

pytestmark = pytest.mark.gpu


def _binding():
    from paper_2602_16603_amd import binding
    return binding


@pytest.mark.parametrize("bad_query", [math.nan, math.inf])
@pytest.mark.parametrize("bad_key", [math.inf, -math.inf])
@pytest.mark.parametrize("latent,rope,heads", [(512, 64, 20), (128, 32, 4), (256, 64, 65)])
@pytest.mark.parametrize("new,cached", [([1], [100]), ([3], [900])])
@pytest.mark.parametrize("workspace", [True, 0])
def test_attention_a_query_that_is_not_finite_beside_a_missing_block(latent, rope, heads, new, cached, bad_key, bad_query, workspace):
    """Block 1 is not there, and a key of block 0, in the same 32 keys, has an infinity.  The last head's query is not finite; that of the
    others meets the infinity with a score of -infinity, so by their formula, 0 * infinity, they have NaN in its column and nowhere else,
    whatever the last head has."""
    B = _binding()
    column, position = 3, 5
    cache = U.Cache(U.blocks_for(new, cached), latent, rope)
    batch = U.Batch(new, cached, cache.n)
    cache.pool[batch.table[0][0], position, column] = bad_key
    batch.table[0][1] = -1
    q = U.normal((sum(new), heads, latent + rope), 1)
    q[..., column] = -math.copysign(1.0, bad_key) * q[..., column].abs().clamp(min=0.125)
    q[:, -1, 7] = bad_query
    scale = (latent + rope) ** -0.5
    ref, tol = cache.attention(batch, q, scale)
    nan = torch.zeros(ref.shape, dtype=torch.bool)
    nan[..., column], nan[:, -1] = True, True
    assert torch.equal(ref.isnan(), nan)                  # (the definition says what the text above does)
    got = U.attend(B, cache, cache.pool.cuda(), batch, q.cuda(), scale, workspace=workspace)
    U.check(got, ref, tol)
