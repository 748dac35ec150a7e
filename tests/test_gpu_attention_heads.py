"""hb_attention against the oracle for every number of query heads that go together and every size of head, with one piece a sequence and with several."""
import numpy as np
import pytest

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_len", [100, 300])
@pytest.mark.parametrize("dim", [34, 80, 128, 130, 192, 194, 256])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_sizes_of_heads(group, dim, max_len):
    Case(np.random.default_rng(1000 * group + dim), 2, 2, group, dim, 12, max_len, [max_len, max_len - 33], sigma=None).check()


@pytest.mark.parametrize("group,dim", [(1, 20), (2, 20), (4, 34), (8, 10), (1, 130)])
def test_many_sequences_of_several_pieces(group, dim):
    """More sequences than are cut together: pieces of one size, of several chunks each."""
    rng = np.random.default_rng(group)
    lens = rng.integers(0, 1501, 70)
    lens[:4] = 0, 1500, 1, 1499
    Case(rng, 70, 2, group, dim, 16, 1500, lens).check()
