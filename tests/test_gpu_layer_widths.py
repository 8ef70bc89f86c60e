"""The layer operators at the widths at which they change their form: every kernel of a row's length, whole vectors and not, and of one and
two rows, compared with the plain binary64 implementation (tests/test_layer_launches.py checks that all of them are reached)."""
import pytest

import test_gpu_layer_ops as ops

pytestmark = pytest.mark.gpu

WIDTHS = [20, 24, 29, 37, 48, 61, 64, 99, 112, 197, 200, 248, 250, 450, 496, 505, 512, 516, 520, 651, 700, 768, 805, 1000, 1021, 1024, 1030, 1096, 1100, 1528,
          1535, 1536, 1544, 1999, 2048, 2052, 2056, 3001, 4000, 4095, 4096, 5000, 7001, 9000, 9001, 16001, 16384, 20000, 20001, 32001, 32768]
WIDE_SIZES = [(1 + i % 7, D, i % 3, i % 2) for i, D in enumerate(WIDTHS)] + [(70, 805, 3, 0), (1031, 1021, 0, 0), (90, 2052, 0, 1), (129, 4095, 1, 0), (600, 768, 0, 0)]


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("M,D,pad,offset", WIDE_SIZES)
def test_layer_norm(dtype, params, M, D, pad, offset):
    ops.test_layer_norm(dtype, params, M, D, pad, offset)


@pytest.mark.parametrize("dtype,params", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("M,D,pad,offset", WIDE_SIZES)
def test_layer_norm_grad(dtype, params, M, D, pad, offset):
    ops.test_layer_norm_grad(dtype, params, M, D, pad, offset)


# One and two rows that go by a launch which reads W once: 64 and 128 bytes of columns to a workgroup, whole vectors of columns and not.
FEW_SIZES = [(1, 2048, 5504), (2, 2048, 5504), (1, 2048, 5503), (2, 1000, 700), (1, 1000, 701), (2, 700, 4099), (1, 700, 4099), (2, 130, 8200), (1, 90, 8201), (2, 90, 8201), (2, 1000, 8203)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F", FEW_SIZES)
def test_one_and_two_rows(dtype, M, D, F):
    ops.test_gated_ff(dtype, M, D, F)


@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_kind_of_step(dtype, grad, bits, copy):
    ops.test_adamw_step(dtype, grad, bits, copy, 1)
