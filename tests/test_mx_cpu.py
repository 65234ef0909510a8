"""Microscaled formats without a GPU: what the oracle's formats mean, the sizes, and what the entry points refuse."""
import ctypes
import subprocess
import sys

import numpy as np
import pytest

from oracle import mx
from paper_2601_22716_b200 import binding as lords
from paper_2601_22716_b200 import build as lords_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    lords_build.build()


def _row(*values):
    v = np.zeros((1, 32))
    v[0, :len(values)] = values
    return v


# ---- the oracle against values worked out by hand ------------------------------------------------------------
def test_four_bit_values_ties_and_limit():
    # the largest value 7 lies in [4, 8): E = 0; 7 is limited to 6, ties go to the even code
    codes, E = mx.quantize4(_row(7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 0.2500001, -6.1))
    assert E.tolist() == [[0]]
    assert codes[0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14, 1, 15]
    assert mx.values4(codes, E)[0, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]


def test_eight_bit_values_ties_and_limit():
    # the largest 1.9921875 = 127.5 / 64 rounds to 128 and is limited to 127; half steps go to the even number
    q, E = mx.quantize8(_row(1.9921875, 1.0, 0.0078125, 0.0234375, -0.0234375, -1.9921875))
    assert E.tolist() == [[0]]
    assert q[0, :6].tolist() == [127, 64, 0, 2, -2, -127]


@pytest.mark.parametrize("below,quantize,values", [(2, mx.quantize4, mx.values4), (0, mx.quantize8, mx.values8)])
def test_exponents_zero_tiny_and_not_finite(below, quantize, values):
    v = np.zeros((4, 70))
    v[1] = 2.0**-133
    v[2, 3], v[2, 40] = np.inf, 1.0
    v[3, 69] = np.nan
    E = mx.exponents(v, below)
    assert E[0].tolist() == [-127] * 3 and E[1].tolist() == [-127] * 3
    assert E[2].tolist() == [128, -below, -127] and E[3].tolist() == [-127, -127, 128]
    out = values(*quantize(v))
    assert (out[0] == 0).all() and np.isnan(out[2, :32]).all() and out[2, 40] == 1.0 and np.isnan(out[3, 64:]).all()


def test_rounding_is_at_most_half_a_step():
    rng = np.random.default_rng(3)
    v = rng.standard_normal((50, 256)) * np.exp(rng.standard_normal((50, 1)))
    codes, E = mx.quantize4(v)
    unit = np.repeat(np.ldexp(1.0, E), 32, axis=1)
    a = np.abs(v) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    err = np.abs(mx.values4(codes, E) - v) / unit
    assert (err <= np.where(a > 6, a - 6, step / 2) + 1e-12).all()
    q, E = mx.quantize8(v)
    assert (np.abs(mx.values8(q, E) - v) <= np.repeat(np.ldexp(1.0, E), 32, axis=1) / 64 * np.where(np.abs(q) == 127, 1.0, 0.5)).all()


# ---- sizes -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (128, 128), (129, 129), (37, 2731), (14336, 4096)])
def test_sizes(rows, cols):
    assert lords.lords_mxfp4_codes_bytes(rows, cols) == rows * ((cols + 31) // 32) * 16
    assert lords.lords_mxfp4_scales_bytes(rows, cols) == (rows + 127) // 128 * ((cols + 127) // 128) * 512
    assert lords.lords_checkpoint_bytes(rows, cols) == rows * ((cols + 31) // 32) * 32
    assert lords.lords_checkpoint_scales_bytes(rows, cols) == rows * ((cols + 127) // 128) * 4


def test_sizes_out_of_range():
    for call in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes, lords.lords_checkpoint_bytes, lords.lords_checkpoint_scales_bytes):
        for rows, cols in ((0, 32), (32, 0), (-1, 4), (2**20 + 1, 32), (32, 2**20 + 1)):
            with pytest.raises(lords.LordsError) as e:
                call(rows, cols)
            assert e.value.status == -2
        assert call(2**20, 2**20) > 2**34       # past 32 bits


# ---- refusals: every check happens on the host, before anything is launched -------------------------------------
A, U = 256, 264          # an aligned and an unaligned address, never followed


def _call(name, *args):
    fn = getattr(ctypes.CDLL(str(lords.library_path())), name)
    fn.restype = ctypes.c_int
    return fn(*[ctypes.c_void_p(a[0]) if isinstance(a, tuple) else a for a in args])


def P(a):
    return (a,)


NULL, SHAPE, ALIGN, BITS, NOT_INIT = -1, -2, -3, -4, -6
_LEVELS = np.zeros(16, dtype=np.float32)
CB = _LEVELS.ctypes.data
TOO = 2**20 + 1

CASES = [
    # lords_mxfp4_quantize(v, rows, cols, codes, scales, codes_t, scales_t, stream)
    ("lords_mxfp4_quantize", (P(0), 4, 4, P(A), P(A), P(A), P(A), P(0)), NULL),
    ("lords_mxfp4_quantize", (P(A), 4, 4, P(0), P(0), P(0), P(0), P(0)), NULL),
    ("lords_mxfp4_quantize", (P(A), 4, 4, P(A), P(0), P(A), P(A), P(0)), NULL),
    ("lords_mxfp4_quantize", (P(A), 4, 4, P(A), P(A), P(0), P(A), P(0)), NULL),
    ("lords_mxfp4_quantize", (P(A), 0, 4, P(A), P(A), P(0), P(0), P(0)), SHAPE),
    ("lords_mxfp4_quantize", (P(A), 4, TOO, P(A), P(A), P(0), P(0), P(0)), SHAPE),
    ("lords_mxfp4_quantize", (P(U), 4, 4, P(A), P(A), P(0), P(0), P(0)), ALIGN),
    ("lords_mxfp4_quantize", (P(A), 4, 4, P(A), P(A), P(A), P(U), P(0)), ALIGN),
    ("lords_mxfp4_quantize", (P(A), 4, 4, P(A), P(A), P(0), P(0), P(0)), NOT_INIT),
    ("lords_mxfp4_dequantize", (P(A), P(0), 4, 4, P(A), P(0)), NULL),
    ("lords_mxfp4_dequantize", (P(A), P(A), 4, -1, P(A), P(0)), SHAPE),
    ("lords_mxfp4_dequantize", (P(A), P(A), 4, 4, P(U), P(0)), ALIGN),
    ("lords_mxfp4_dequantize", (P(A), P(A), 4, 4, P(A), P(0)), NOT_INIT),
    # lords_mxfp4_matmul(x_codes, x_scales, w_codes, w_scales, M, m, n, y, stream)
    ("lords_mxfp4_matmul", (P(A), P(A), P(A), P(0), 1, 1, 1, P(A), P(0)), NULL),
    ("lords_mxfp4_matmul", (P(A), P(A), P(A), P(A), 0, 1, 1, P(A), P(0)), SHAPE),
    ("lords_mxfp4_matmul", (P(A), P(A), P(A), P(A), 1, TOO, 1, P(A), P(0)), SHAPE),
    ("lords_mxfp4_matmul_f32", (P(A), P(A), P(A), P(A), 1, 1, 0, P(A), P(0)), SHAPE),
    ("lords_mxfp4_matmul_f32", (P(A), P(U), P(A), P(A), 1, 1, 1, P(A), P(0)), ALIGN),
    ("lords_mxfp4_matmul", (P(A), P(A), P(A), P(A), 1, 1, 1, P(A), P(0)), NOT_INIT),
    ("lords_mxfp4_forward", (P(0), P(A), P(A), 1, 1, 1, P(A), P(0)), NULL),
    ("lords_mxfp4_forward", (P(A), P(A), P(A), 1, 1, TOO, P(A), P(0)), SHAPE),
    ("lords_mxfp4_forward_f32", (P(A), P(A), P(A), 1, 1, 1, P(U), P(0)), ALIGN),
    ("lords_mxfp4_forward_f32", (P(A), P(A), P(A), 1, 1, 1, P(A), P(0)), NOT_INIT),
    ("lords_checkpoint_store", (P(A), 4, 4, P(A), P(0), P(0)), NULL),
    ("lords_checkpoint_store", (P(A), 4, 0, P(A), P(A), P(0)), SHAPE),
    ("lords_checkpoint_store", (P(A), 4, 4, P(U), P(A), P(0)), ALIGN),
    ("lords_checkpoint_store", (P(A), 4, 4, P(A), P(A), P(0)), NOT_INIT),
    ("lords_checkpoint_load", (P(0), P(A), 4, 4, P(A), P(0)), NULL),
    ("lords_checkpoint_load", (P(A), P(A), TOO, 4, P(A), P(0)), SHAPE),
    ("lords_checkpoint_load", (P(A), P(U), 4, 4, P(A), P(0)), ALIGN),
    ("lords_checkpoint_load", (P(A), P(A), 4, 4, P(A), P(0)), NOT_INIT),
    # ..._factors_checkpoint(dy, q, e, Qpacked, B, A, codebook, bits, M, m, n, r, dB, dA, stream)
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(0), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(A), P(A), P(0)), NULL),
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(0), P(0), P(0)), NULL),
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 5, 2, 4, 4, 2, P(A), P(A), P(0)), BITS),
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 3, 2, P(A), P(A), P(0)), SHAPE),
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 129, P(A), P(A), P(0)), SHAPE),
    ("lords_linear_backward_factors_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(A), P(A), P(0)), NOT_INIT),
    # ..._qat_checkpoint(dy, q, e, W, Qpacked, B, A, codebook, bits, M, m, n, r, dW, dB, dA, stream)
    ("lords_linear_backward_qat_checkpoint", (P(A), P(0), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(A), P(A), P(A), P(0)), NULL),
    ("lords_linear_backward_qat_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 0, 4, 4, 2, P(A), P(A), P(A), P(0)), SHAPE),
    ("lords_linear_backward_qat_checkpoint", (P(A), P(U), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(A), P(A), P(A), P(0)), ALIGN),
    ("lords_linear_backward_qat_checkpoint", (P(A), P(A), P(A), P(A), P(A), P(A), P(A), P(CB), 4, 2, 4, 4, 2, P(A), P(A), P(A), P(0)), NOT_INIT),
]


@pytest.mark.parametrize("name,args,status", CASES, ids=[f"{k}-{c[0]}-{c[2]}" for k, c in enumerate(CASES)])
def test_refusals(name, args, status):
    if status == NOT_INIT:          # in a process of its own: another test may have bound the library
        code = f"import ctypes\nf = getattr(ctypes.CDLL({str(lords.library_path())!r}), {name!r})\nP = lambda a: (a,)\n" \
               f"import numpy as np\nt = np.zeros(16, dtype=np.float32)\nargs = {args!r}\n" \
               "assert f(*[ctypes.c_void_p(a[0]) if isinstance(a, tuple) else a for a in args]) == -6"
        code = code.replace(repr((CB,)), "(t.ctypes.data,)")
        subprocess.run([sys.executable, "-c", code], check=True)
    else:
        assert _call(name, *args) == status
