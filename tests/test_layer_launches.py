"""What layer operators launch at the largest sizes that they accept, and which forms they take: the host code runs against a recorder
of launches (tests/launch_lanes.c), so nothing of that size has to exist.  CPU only."""
import json
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2311_16883_amd import binding as B

HERE = Path(__file__).resolve().parent
LIB = HERE.parent / "paper_2311_16883_amd" / "libbsr_actprune.so"
F32, BF16 = 0, 1
MOST, WIDE = (1 << 31) - 1, 1 << 20


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    so = tmp_path_factory.mktemp("recorder") / "liblaunch_lanes.so"
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(so), str(HERE / "launch_lanes.c")], check=True)
    B.lib()                                          # built if it is not there yet
    return so


def run(recorder, program, *calls):
    r = subprocess.run([sys.executable, str(HERE / program), str(recorder), str(LIB)], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def norm(M, D, dtype=BF16):
    return ["bsr_layer_norm", ["p", dtype, M, D, D, "p", "p", F32, 1e-5, "p", D, "p", None]]


def norm_grad(M, D, dtype=BF16):
    return ["bsr_layer_norm_grad", ["p", dtype, M, D, D, "p", F32, "p", "p", D, "p", D, "p", "p", 0, "ws", None]]


def gated(M, D, F, dtype=BF16, ldw=None):
    return ["bsr_gated_ff", ["p", dtype, M, D, D, "p", F, ldw or 2 * F, 0, "p", F, "p", 2 * F, "ws", None]]


def gated_grad(M, D, F, dtype=BF16):
    return ["bsr_gated_ff_grad", ["p", dtype, M, F, 2 * F, "p", F, 1, "p", D, 2 * F, "p", 2 * F, "p", D, "ws", None]]


LARGEST = [norm(MOST, 1), norm(MOST, 64), norm(MOST, 2048), norm(MOST, 1 << 20), norm(3, MOST), norm(MOST, 5, F32),
           norm_grad(MOST, 1), norm_grad(MOST, 64), norm_grad(MOST, 2048), norm_grad(MOST, 9000), norm_grad(MOST, 1 << 20), norm_grad(3, MOST), norm_grad(1, MOST, F32),
           gated(MOST, 1, 1), gated(MOST, 8, 8), gated(MOST, 64, 4096), gated(1, WIDE, WIDE // 2), gated(20, WIDE, WIDE // 2), gated(1000, WIDE, WIDE // 2, F32),
           gated(MOST, 40, 40, F32), gated(1 << 20, 1000, WIDE // 2), gated(2, WIDE, 9),
           gated_grad(MOST, 1, 1), gated_grad(MOST, 64, 64), gated_grad(1 << 23, WIDE, 64), gated_grad(7, WIDE, WIDE // 2), gated_grad(MOST, 40, 41, F32)]


@pytest.mark.parametrize("i", range(len(LARGEST)), ids=lambda i: "%s-%d" % (LARGEST[i][0], i))
def test_launches_of_the_largest_sizes_are_ones_that_the_hardware_takes(recorder, i):
    """Lanes along a dimension are counted in 32 bits, workgroups along the second and third in 16."""
    got, = run(recorder, "recorded_token_calls.py", LARGEST[i])
    assert got["rc"] == 0 and got["launches"]
    for l in got["launches"]:
        assert all(0 < n < 1 << 32 for n in l["lanes"]), l
        assert l["grid"][1] < 1 << 16 and l["grid"][2] < 1 << 16, l


def test_every_tile_of_the_most_rows_has_a_workgroup(recorder):
    for M, D, F, area in ((MOST, 64, 4096, None), (1 << 26, 200, 40, None)):
        got, = run(recorder, "recorded_token_calls.py", gated(M, D, F))
        parts = [l for l in got["launches"] if "product_kernel" in l["kernel"]]
        assert len(got["launches"]) == len(parts)
        # a wave has 64 lanes and at most 128 rows x 32 columns of H
        assert sum(l["lanes"][0] for l in parts) >= M * F * 64 // (128 * 32)


@pytest.mark.parametrize("sizes,bits", [([1 << 40], 8), ([1 << 40], 32), ([5, 1 << 36, 7, (1 << 33) + 3], 8), ([3] * 100, 32), ([], 8), ([0, 0], 8)])
def test_every_element_of_an_optimizer_step_has_a_lane(recorder, sizes, bits):
    got, = run(recorder, "recorded_adamw_calls.py", [sizes, bits])
    assert got["rc"] == 0
    assert all(0 < l["lanes"] < 1 << 32 for l in got["launches"])
    # a workgroup of 256 lanes takes one or four rounds of at most eight elements a lane
    assert sum(l["lanes"] for l in got["launches"]) * 32 >= sum(sizes)
    assert len(got["launches"]) <= 1 + sum(sizes) / (1 << 32) + len(sizes) / 20


def kernels(recorder, call):
    got, = run(recorder, "recorded_token_calls.py", call)
    assert got["rc"] == 0
    return [l["kernel"] for l in got["launches"]]


def test_operands_are_copied_only_where_their_rows_are_no_whole_words(recorder):
    """The copies of the tests' odd sizes: bfloat16 rows that start between words, in one launch (beside the slopes on the way back)."""
    for dtype, D, F, packs in ((BF16, 128, 64, 0), (BF16, 66, 34, 0), (BF16, 65, 64, 1), (BF16, 64, 33, 1), (F32, 65, 33, 0), (F32, 63, 1, 0)):
        names = kernels(recorder, gated(300, D, F, dtype))
        assert sum("pack_kernel" in n for n in names) == packs, names
    assert len(kernels(recorder, gated_grad(300, 64, 33))) == len(kernels(recorder, gated_grad(300, 64, 32)))


def test_one_and_two_rows_are_one_launch(recorder):
    for M in (1, 2):
        assert len(kernels(recorder, gated(M, 1000, 700))) == 1
        assert "gated_few_kernel" in kernels(recorder, gated(M, 1000, 701))[0]
    assert any("product_kernel" in k for k in kernels(recorder, gated(1, 1000, 3, F32)))    # (fewer columns than a vector)


def test_up_to_32_rows_are_one_launch_where_that_is_faster(recorder):
    for M, D, F in ((3, 1000, 704), (32, 2048, 5504), (16, 1000, 701), (1, 1000, 7)):
        names = kernels(recorder, gated(M, D, F))
        assert len(names) == 1 and "gated_rows_kernel" in names[0], names
    for M, D, F in ((33, 1000, 700), (8, 8192, 1024), (8, 256, 16384), (3, 64, 64)):
        assert "product_kernel" in kernels(recorder, gated(M, D, F))[0]


def test_sizes_of_the_gpu_tests_reach_every_product_kernel(recorder):
    from test_gpu_layer_ops import GATED_SIZES, TILE_GRAD_SIZES, TILE_SIZES
    reached = set()
    for dtype in (BF16, F32):
        for sizes, call in ((GATED_SIZES + TILE_SIZES, gated), (GATED_SIZES + TILE_GRAD_SIZES, gated_grad)):
            for size in sizes:
                reached |= {n for n in kernels(recorder, call(*size, dtype)) if "product_kernel" in n}
    there = {n for n in subprocess.run(["nm", str(LIB)], capture_output=True, text=True, check=True).stdout.split() if "product_kernel" in n}
    there = {n for n in there if "__device_stub__" not in n}
    assert reached and reached <= there
    assert sorted(there - reached) == []


def test_few_rows_of_a_norm_leave_nothing_to_add_up(recorder):
    assert len(kernels(recorder, norm_grad(8, 384))) == 1
    assert len(kernels(recorder, norm_grad(100, 384))) == 2


def norm_grad_alone(M, D, dtype=BF16):
    """... without the gradients of weight and bias"""
    name, args = norm_grad(M, D, dtype)
    return [name, args[:12] + [None, None] + args[14:]]


def test_sizes_of_the_gpu_tests_reach_every_norm_kernel_and_those_of_few_rows(recorder):
    """Sizes whose results the GPU tests compare with the plain implementation."""
    from test_gpu_layer_ops import NORM_SIZES
    from test_gpu_layer_widths import FEW_SIZES, WIDE_SIZES
    calls = []
    for dtype in (BF16, F32):
        for M, D, _, _ in NORM_SIZES + WIDE_SIZES:
            calls += [norm(M, D, dtype), norm_grad(M, D, dtype), norm_grad_alone(M, D, dtype)]
        calls += [gated(*size, dtype) for size in FEW_SIZES]
        calls.append(norm_grad(0, 5, dtype))
    reached = {l["kernel"] for got in run(recorder, "recorded_token_calls.py", *calls) for l in got["launches"]}
    kinds = ("layer_norm", "gated_few_kernel", "gated_rows_kernel", "clear_sums_kernel")
    symbols = subprocess.run(["nm", str(LIB)], capture_output=True, text=True, check=True).stdout.split()
    there = {n for n in symbols if any(k in n for k in kinds) and "_kernel" in n and "__device_stub__" not in n}
    assert len(there) > 100 and sorted(there - reached) == []
