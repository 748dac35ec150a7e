"""How linear layers are shared out to workgroups and dies (no GPU)."""
import numpy as np
import pytest

import linear_cases
from plan_util import plan

DIES = 8


@pytest.mark.parametrize("count", [1, 2, 7, 8, 9, 15, 16, 17, 63, 64, 65, 256, 1000, 1024, 4099])
def test_every_pair_once_and_all_dies_alike(count):
    """Workgroup b runs on die b mod 8."""
    pairs = np.array([plan().pair(b, count) for b in range(count)])
    assert sorted(pairs) == list(range(count))
    loads = [len(pairs[die::DIES]) for die in range(DIES)]
    assert max(loads) - min(loads) <= 1
    for die in range(DIES):                                          # an eighth of the pairs, in order
        assert np.array_equal(pairs[die::DIES], pairs[die: die + 1].repeat(loads[die]) + np.arange(loads[die]))


@pytest.mark.parametrize("rows,outs", [(2048, 1024), (2048, 256), (2048, 128), (48, 640), (64, 16384), (16, 4096), (1, 4096), (5, 1411), (1, 1)])
@pytest.mark.parametrize("flush", [32, 64, 128])
def test_rounds_are_those_that_the_price_counts(rows, outs, flush):
    """The fullest die's 32 compute units go round as often as 256 of the whole card would."""
    form = plan().form(flush, rows, outs)
    count = plan().row_tiles(form, rows) * plan().groups(form, outs)
    fullest = -(-count // DIES)
    assert -(-fullest // 32) == -(-count // 256)


def test_many_groups_stay_on_a_die():
    """64 x (4096 -> 16384): a group's weights are read by one die's workgroups alone."""
    rows, outs = 64, 16384
    form = plan().form(128, rows, outs)
    tiles, groups = plan().row_tiles(form, rows), plan().groups(form, outs)
    count = tiles * groups
    group_of = np.array([plan().pair(b, count) for b in range(count)]) // tiles
    dies = {}
    for b, g in enumerate(group_of):
        dies.setdefault(int(g), set()).add(b % DIES)
    assert len(dies) == groups and all(len(d) == 1 for d in dies.values())


@pytest.mark.parametrize("rows,outs", [(1 << 24, 1), (1 << 24, 16), (1 << 24, 1 << 24), (1, 1 << 24), (1 << 23, 128), ((1 << 21) - 1, 16), (1 << 22, 1000)])
@pytest.mark.parametrize("flush", [32, 64, 128])
def test_grids_of_the_largest_sizes(rows, outs, flush):
    """Every size up to the stated limits has launches, each of fewer than 2^32 threads."""
    form = plan().form(flush, rows, outs)
    tiles, groups = plan().row_tiles(form, rows), plan().groups(form, outs)
    assert tiles < 1 << 32
    for threads in (256, 512, 1024):
        most = plan().launch_tiles(groups, threads)
        assert most >= 3 and most * groups * threads < 1 << 32 <= (most + 1) * groups * threads


@pytest.mark.parametrize("form,rows,inputs,outs,group", linear_cases.cases())
def test_the_gpu_tests_reach_the_forms_that_they_say(form, rows, inputs, outs, group):
    assert plan().form(group, rows, outs) == form


def test_every_form_has_cases():
    for group in linear_cases.GROUPS:
        assert {case[0] for case in linear_cases.cases() if case[4] == group} == set(range(8 if group == 32 else 9))


def test_one_row_of_many_outputs():
    """The form that shares one row's digits among four tiles is taken where it is the fastest: 9000 to 16384 outputs 9.0 to 11.3 us for 10.0 to 12.1 with the next
    one, to 49152 20.0 to 30.8 for 21.3 to 32.0; from 57000 on (34.6 and 38.2) eight tiles are shared."""
    for outs in (9000, 12288, 16384, 24576, 32768, 40000, 49152, 81920):
        assert plan().form(128, 1, outs) == plan().form(64, 1, outs) == 8, outs
    for outs in (57000, 65536, 98304, 131072, 200000):
        assert plan().form(128, 1, outs) == 5, outs
    assert plan().form(128, 1, 8192) == 2 and plan().form(128, 1, 4096) == 0
