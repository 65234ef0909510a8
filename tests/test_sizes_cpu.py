"""Sizes that no C int holds, in every call that takes tensors: refused as a negative size is.  (Each call ends in its
checks: the library is not bound to a device, and the process sees none.)"""
import os
import subprocess
import sys

import pytest

from paper_2601_22716_b200 import build as lords_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    lords_build.build()


# name -> arguments in order: "p" a tensor, "c" the level table, else a size with a value that the call takes
FORWARD = ("p", "p", "p", "p", "c", ("bits", 4), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p")
CALLS = {
    "lords_linear_forward": ("p", "p", "p", "p", "c", ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p"),
    "lords_linear_forward_bits": FORWARD,
    "lords_linear_forward_f32": FORWARD,
    "lords_linear_forward_host": FORWARD,
    "lords_linear_forward_noalloc": FORWARD,
    "lords_linear_backward_input": FORWARD,
    "lords_linear_backward_input_f32": FORWARD,
    "lords_quantize_codes": ("p", "p", "p", "c", ("bits", 4), ("m", 64), ("n", 64), ("r", 4), "p"),
    "lords_transpose_codes": ("p", ("bits", 4), ("m", 64), ("n", 64), "p"),
    "lords_linear_backward_factors": ("p", "p", "p", "p", "p", "c", ("bits", 4), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p", "p"),
    "lords_linear_backward_qat": ("p", "p", "p", "p", "p", "p", "c", ("bits", 4), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p", "p", "p"),
    "lords_blockscale_forward": ("p", "p", "p", "c", ("bits", 4), ("blk", 64), ("M", 2), ("m", 64), ("n", 64), "p"),
    "lords_adapter_forward": ("p", "p", "p", "p", "p", "c", ("bits", 4), ("blk", 64), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p"),
    "lords_mxfp4_quantize": ("p", ("rows", 4), ("cols", 64), "p", "p"),
    "lords_mxfp4_dequantize": ("p", "p", ("rows", 4), ("cols", 64), "p"),
    "lords_mxfp4_matmul": ("p", "p", "p", "p", ("M", 2), ("m", 64), ("n", 64), "p"),
    "lords_mxfp4_forward": ("p", "p", "p", ("M", 2), ("m", 64), ("n", 64), "p"),
    "lords_checkpoint_store": ("p", ("M", 4), ("n", 64), "p", "p"),
    "lords_checkpoint_load": ("p", "p", ("M", 4), ("n", 64), "p"),
    "lords_linear_backward_factors_checkpoint": ("p", "p", "p", "p", "p", "p", "c", ("bits", 4), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p", "p"),
    "lords_linear_backward_qat_checkpoint": ("p", "p", "p", "p", "p", "p", "p", "c", ("bits", 4), ("M", 2), ("m", 64), ("n", 64), ("r", 4), "p", "p", "p"),
}

SCRIPT = """
import numpy as np
from paper_2601_22716_b200 import binding as lords

class Tensor:                 # an address that is never followed
    is_cuda = False
    def data_ptr(self):
        return 4096

class Stream:
    cuda_stream = 0

NAME, SPEC = {name!r}, {spec!r}
TABLE = np.linspace(-1, 1, 16, dtype=np.float32)

def outcome(which, value):
    args = [Tensor() if a == "p" else TABLE if a == "c" else value if a[0] == which else a[1] for a in SPEC]
    try:
        getattr(lords, NAME)(*args, stream=Stream())
    except lords.LordsError as e:
        return "status", e.status
    except ValueError:
        return ("ValueError",)         # the level table does not have 2**bits entries
    return ("accepted",)

assert outcome(None, None) in (("status", -6), ("status", -7))          # every size as it is: only the device is missing
for which in [a[0] for a in SPEC if a not in ("p", "c")]:
    want = outcome(which, -1)
    for value in (2**31, 2**31 + 4, 2**32, 2**32 + 4, 2**32 + 64, 2**40, 2**63, 2**70, -2**31 - 1, -2**40, -2**70):
        got = outcome(which, value)
        assert got == want, (which, value, got, want)
"""


@pytest.mark.parametrize("name", CALLS)
def test_sizes_that_no_int_holds(name):
    subprocess.run([sys.executable, "-c", SCRIPT.format(name=name, spec=CALLS[name])], check=True, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
