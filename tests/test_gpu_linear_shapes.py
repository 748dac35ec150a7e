"""hb_linear_q4 against the oracle in every form of its kernel, and where rows and outputs are far apart."""
import numpy as np
import pytest

import decode_util as du
import linear_cases
from oracle import decode
from paper_2309_04875_amd import hb

pytestmark = pytest.mark.gpu
SEED = 0x2309048750000061


def check(rng, rows, inputs, outputs, group, frac=18, sigma=1.0, big=False):
    x, weight, scales = du.layer(rng, rows, inputs, outputs, group, frac, sigma, big)
    o0, o1, bits = hb.hb_linear_q4(*du.gpu(*x, weight, scales), group, frac, SEED)
    assert bits == 64 * rows * outputs
    for got, want in zip((o0, o1), decode.linear(*x, weight, scales, group, frac, SEED)):
        bad = np.argwhere(du.host(got) != want)
        assert got.shape == want.shape and not len(bad), "%d of %d differ, first at %s" % (len(bad), want.size, bad[0])


@pytest.mark.parametrize("rows,inputs,outputs,group", [(300, 70, 16, 32), (2049, 40, 1, 64), (1031, 300, 100, 128), (2051, 260, 250, 128), (48, 1000, 640, 128),
                                                       (530, 129, 1025, 32)])
def test_many_rows_of_few_outputs(rows, inputs, outputs, group):
    """Fewer groups of outputs than dies, or a remainder of them."""
    check(np.random.default_rng(rows), rows, inputs, outputs, group)


@pytest.mark.parametrize("rows,inputs,outputs,group", [(1 << 24, 1, 1, 32), ((1 << 21) + 3, 2, 17, 64)])
def test_as_many_rows_as_there_may_be(rows, inputs, outputs, group):
    """More workgroups than one grid holds; and a size that was refused when a layer's groups were rounded up to the number of dies."""
    check(np.random.default_rng(9), rows, inputs, outputs, group)


@pytest.mark.parametrize("form,rows,inputs,outputs,group", linear_cases.cases())
def test_every_form(form, rows, inputs, outputs, group):
    """Inputs over all 64 bits, scales over all of int32."""
    check(np.random.default_rng(100 * form + group), rows, inputs, outputs, group, 20, None, True)
