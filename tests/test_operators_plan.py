"""The linear cross entropy's host arithmetic (pieces, tiles, slots, workspace) without a GPU: every extent of a call lies in its
buffer, over random sizes and over sizes at which one did not."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", lib, os.path.join(HERE, "xent_plan_check.cpp")], check=True)
    return ctypes.CDLL(lib)


@pytest.mark.parametrize("max_rows,rows,features,classes", [(3500, 3500, 4096, 32768), (3500, 3500, 4096, 131072), (3329, 3329, 4096, 32768),
                                                            (3584, 3584, 2048, 32768), (5632, 4864, 4096, 32768), (3584, 3584, 4096, 128256),
                                                            (3584, 3584, 8192, 100000)])
def test_pairs_of_weights_that_are_copied_fit(plan, max_rows, rows, features, classes):
    """Pieces of the classes are tiled each for itself: more slots than one tiling of all of them has."""
    for grad in (0, 1):
        for direct in (0, 1):
            assert plan.check_call(max_rows, rows, features, classes, BF16, direct, grad, 74) == 1


@pytest.mark.parametrize("rows,features,classes,direct", [(3072, 64, 44544, 1), (546, 3600, 12750, 0), (3072, 64, 44544, 0)])
def test_the_last_piece_reads_no_bias_behind_its_end(plan, rows, features, classes, direct):
    assert plan.check_call(rows, rows, features, classes, BF16, direct, 1, 74) == 1


@pytest.mark.parametrize("pairs", [74, 66, 9])
def test_every_extent_of_random_calls_lies_in_its_buffer(plan, pairs):
    assert plan.sweep(pairs, 200000, pairs) == 0


def test_every_number_of_rows_at_some_sizes(plan):
    for features, classes in ((4096, 32768), (2048, 50021), (1001, 20000), (72, 600000)):
        for kind in (F32, BF16, F16):
            for rows in range(1, 9000, 61):
                assert plan.check_call(rows, rows, features, classes, kind, 0, 1, 74) == 1
                assert plan.check_call(9000, rows, features, classes, kind, 0, 0, 74) == 1
