"""What token operators launch at the largest sizes that they accept: the host code runs against a recorder of launches
(tests/launch_lanes.c), so nothing of that size has to exist.  CPU only."""
import json
import re
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2311_16883_amd import binding as B

HERE = Path(__file__).resolve().parent
LIB = HERE.parent / "paper_2311_16883_amd" / "libbsr_actprune.so"
F32, BF16, I32, I64 = 0, 1, 0, 1
MOST = (1 << 31) - 1                                 # rows, positions, entries


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    so = tmp_path_factory.mktemp("recorder") / "liblaunch_lanes.so"
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(so), str(HERE / "launch_lanes.c")], check=True)
    B.lib()                                          # built if it is not there yet

    def run(*calls):
        r = subprocess.run([sys.executable, str(HERE / "recorded_token_calls.py"), str(so), str(LIB)], input=json.dumps(calls),
                           capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)

    return run


def lookup(T, V, D, dtype=BF16):
    return ["bsr_embedding_lookup", ["p", dtype, V, D, D, "p", I32, T, 1.0, "p", D, None]]


def table_grad(T, V, D, dtype=BF16, accumulate=0, ldde=None):
    return ["bsr_embedding_grad", ["p", I32, T, "p", dtype, D, D, 1.0, V, "p", ldde or D, accumulate, "ws", None]]


def expert_sort(n, E, align=1):
    return ["bsr_expert_sort", ["p", I32, n, E, align, "p", "p", "p", "p", "ws", None]]


def gather(T, k, rows, D):
    return ["bsr_expert_gather", ["p", BF16, T, D, D, "p", k, "p", rows, "p", D, None]]


def combine(T, k, rows, D):
    return ["bsr_expert_combine", ["p", BF16, rows, D, D, "p", T, k, None, "p", D, None]]


def combine_grad(T, k, rows, D):
    return ["bsr_expert_combine_grad", ["p", BF16, rows, D, D, "p", "p", T, k, "p", "p", D, "p", D, "p", None]]


def distill_grad(N, V, K):
    return ["bsr_distill_grad", ["p", BF16, N, V, V, "p", I32, "p", BF16, K, 1.0, "p", "p", "p", V, None]]


def distill_both(N, V, K):
    return ["bsr_distill_loss_grad", ["p", BF16, N, V, V, "p", I32, "p", BF16, K, 1.0, "p", "p", "p", V, "ws", None]]


LARGEST = [
    lookup(MOST, MOST, 1), lookup(MOST, 1000, 1024), lookup(MOST, 5, 8, F32),
    table_grad(MOST, 1000, 1), table_grad(MOST, 1000, 8), table_grad(MOST, 1000, 3, F32), table_grad(MOST, 1000, 1, BF16, 1),
    table_grad(MOST, 1, 1), table_grad(MOST - 31, (1 << 30) - 1, 1), table_grad(1 << 30, 50000, 512),
    table_grad(1, (1 << 30) - 1, 64), table_grad(9000, (1 << 30) - 1, 3, F32, 0, 7),
    expert_sort(MOST, 1024), expert_sort(MOST - 5, 1), expert_sort(1000, 7, 1 << 28),
    gather(MOST, 1, MOST, 1), gather(1 << 28, 7, MOST, 512), combine(MOST, 1, MOST, 1), combine(1 << 28, 7, MOST, 512),
    combine_grad(MOST, 1, MOST, 1), combine_grad(1 << 28, 7, MOST, 512),
    distill_grad(1 << 27, 40, 3), distill_grad(2, MOST, 3), distill_both(1 << 27, 40, 3), distill_both(2, MOST, 3),
    distill_both(1 << 20, 60000, 3), distill_both(70000, 600000, 3),
]


@pytest.mark.parametrize("i", range(len(LARGEST)), ids=lambda i: "%s-%d" % (LARGEST[i][0], i))
def test_launches_of_the_largest_sizes_are_ones_that_the_hardware_takes(record, i):
    """Lanes along a dimension are counted in 32 bits, workgroups along the second and third in 16."""
    got, = record(LARGEST[i])
    assert got["rc"] == 0 and got["launches"]
    for l in got["launches"]:
        assert all(0 < n < 1 << 32 for n in l["lanes"]), l
        assert l["grid"][1] < 1 << 16 and l["grid"][2] < 1 << 16, l


def test_every_position_of_the_largest_table_gradient_has_a_wave(record):
    for T, size in ((MOST, 62), ((1 << 30) + 1, 62), (1 << 30, 32), (100000, 32)):
        got, = record(table_grad(T, 1000, 1))
        sums = [l for l in got["launches"] if "window_sum_kernel" in l["kernel"]]
        joins = [l for l in got["launches"] if "join_kernel" in l["kernel"]]
        windows = -(-T // size)
        assert len(sums) == len(joins) == 1
        assert sums[0]["lanes"][0] * sums[0]["lanes"][1] >= windows * 64
        assert joins[0]["grid"][0] * joins[0]["grid"][1] >= -(-windows // 4)


def forms(got, kernel):
    """The truth values among the template arguments of a launched kernel: whether it reads and writes past the caches."""
    names = [l["kernel"] for l in got["launches"] if kernel in l["kernel"]]
    assert len(names) == 1, got
    return [c == "1" for c in re.findall(r"Lb([01])E", names[0])]


MIB = 1 << 20


def test_rows_pass_by_the_caches_from_the_stated_sizes_on(record):
    """32 MiB written, 64 MiB read, 96 MiB of a table's gradients, in rows of whole 128-byte lines: what the tests of these sizes on the
    GPU (test_gpu_token_large.py) mean to reach."""
    D, row = 1024, 2048
    for T, yes in ((32 * MIB // row, True), (32 * MIB // row - 1, False)):
        got, = record(lookup(T, 3000, D))
        assert forms(got, "embedding_lookup_kernel") == [yes]
        got, = record(gather(T // 2 - 40, 2, T, D))
        assert forms(got, "expert_gather_kernel") == [yes]
    got, = record(lookup(32 * MIB // row + 100, 3000, D - 8))
    assert forms(got, "embedding_lookup_kernel") == [False]
    for T, rows, k, want in ((16384, 32768, 3, [True, True]), (16383, 32768, 2, [True, False]), (16384, 32767, 5, [False, True]),
                             (16383, 32767, 1, [False, False])):
        got, = record(combine(T, k, rows, D))
        assert forms(got, "expert_combine_kernel") == want
    for rows, want in ((32768, [True, True]), (32767, [False, True]), (16384, [False, True]), (16383, [False, False])):
        got, = record(combine_grad(rows // 2, 2, rows, D))
        assert forms(got, "expert_combine_grad_kernel") == want
    for T, yes in ((96 * MIB // row, True), (96 * MIB // row - 1, False)):
        got, = record(table_grad(T, 5000, D))
        assert forms(got, "window_sum_kernel") == [yes]
