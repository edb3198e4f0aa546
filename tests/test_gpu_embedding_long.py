"""The embedding's gradient of texts whose sorted chunks are merged in several passes, against double precision with the bounds of
test_gpu_embedding.py (a row's k gradients in any order: k u of their magnitudes)."""
import pytest

from test_gpu_embedding import _check_backward, _rand, _tokens

pytestmark = pytest.mark.gpu


# 64 chunks of 16384 tokens are merged in one pass; one token more makes a chunk and a group of its own
@pytest.mark.parametrize("kind", ["text", "stray", "one"])
@pytest.mark.parametrize("n,rows,vocab", [(1, 1_048_576, 1000), (1, 1_048_577, 100_003), (2, 1_100_001, 301)])
def test_passes_of_merging(n, rows, vocab, kind):
    _check_backward(_tokens(n, rows, vocab, rows, kind), _rand((n, rows, 4), 1.0, 3, "bf16"), vocab, "f32", 0.5)
