"""Copies of a plan that scans have used: the programs laid out for it, which hold addresses of device memory, do not go with them."""
import copy
import dataclasses
import pickle

import numpy as np
import pytest

import paper_2511_00413_amd as T
from paper_2511_00413_amd import binding as B


def used_plan():
    plan = T.tree_gdn_plan([-1, 0, 0], [130, 70, 65], [1])
    plan._scan_program(64, False)
    plan.scan_programs[(64, False, "a device")] = ("tensor", B._ScanChunks(3, 1), B._ScanChunks(3, 1), 0)      # as a call leaves it
    return plan


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda p: pickle.loads(pickle.dumps(p)), dataclasses.replace])
def test_copies(how):
    plan = used_plan()
    other = how(plan)
    assert not other.scan_programs and plan.scan_programs
    assert np.array_equal(other._scan_program(64, False), plan._scan_program(64, False)) and len(other.scan_programs) == 1


def test_a_changed_plan_is_laid_out_anew():
    """The same tree, another node captured."""
    plan, want = used_plan(), T.tree_gdn_plan([-1, 0, 0], [130, 70, 65], [0])
    other = dataclasses.replace(plan, chunk_cap=want.chunk_cap)
    assert np.array_equal(other._scan_program(64, False), want._scan_program(64, False))
    assert not np.array_equal(other._scan_program(64, False), plan._scan_program(64, False))


def test_the_fields_of_a_used_plan():
    plan = used_plan()
    assert dataclasses.asdict(plan).keys() == dataclasses.asdict(T.tree_gdn_plan([-1], [3])).keys() and "scan" not in repr(plan)
