"""Products per head of many tokens whose workgroups take runs of several rounds, ended inside one of them."""
import pytest

from tests import test_gpu_latent as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,heads,n,k", [
    (700, 64, 128, 512),       # two rounds to a run, the last run of 188 tokens
    (1300, 64, 128, 512),      # three
    (1025, 128, 64, 64),       # five, the last run of 385
    (300, 256, 8, 64),         # one run
    (70, 300, 24, 256),        # one round, some of its waves without tokens
    (520, 60, 600, 128),       # two tiles of outputs
    (40, 1000, 16, 64),        # most waves without tokens
])
def test_runs_of_several_rounds(m, heads, n, k):
    L.test_gemm_heads_matches_the_definition(m, heads, n, k)
