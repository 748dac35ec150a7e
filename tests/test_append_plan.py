"""How appended tokens are shared out to launches (no GPU)."""
import pytest

from plan_util import plan

MOST = 1 << 24                                                      # tokens of a call


@pytest.mark.parametrize("heads,q_heads,dim", [(1, 0, 2), (1, 129, 2), (1, 0, 256), (8, 32, 128), (12, 12, 80), (4096, 65536, 256), (4096, 0, 256), (3, 5, 130)])
@pytest.mark.parametrize("n", [1, 2])
def test_every_launch_fits_a_grid(heads, q_heads, dim, n):
    groups = dim // (2 * n)                                         # of a head
    if groups == 0:
        return
    stored, asked = heads * groups, q_heads * groups
    most = plan().append_tokens(stored, asked)
    assert most >= 256

    def threads(tokens):
        return 256 * (2 * plan().append_blocks(tokens, stored) + plan().append_blocks(tokens, asked))
    for tokens in (1, 2, most - 1, most, MOST % most, MOST - most):
        if 0 < tokens <= most:
            assert 0 < threads(tokens) < 1 << 32
    assert most >= MOST or threads(most) > 1 << 30                   # and no more launches than there have to be


def test_ordinary_calls_are_one_launch():
    for heads, q_heads, dim in ((8, 32, 128), (12, 12, 80), (1, 8, 64)):
        assert plan().append_tokens(heads * dim // 4, q_heads * dim // 4) > 100000
