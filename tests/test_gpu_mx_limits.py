"""Microscaled formats at the ends of their ranges, and a process whose first calls come from several threads at once."""
import subprocess
import sys

import pytest
import torch

from paper_2601_22716_b200 import binding as lords

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    lords.lords_init(0, 0)
    yield
    torch.cuda.synchronize()
    assert lords.lords_poll_status() == 0
    lords.lords_shutdown()


GUARD = 0xA5


def _bytes(count):
    whole = torch.full((count + 256,), GUARD, dtype=torch.uint8, device="cuda")
    return whole[:count], whole[count:]


def _four(rows, cols):
    return [torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes)]


def _normal(rows, cols, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols, generator=gen, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("rows", [1 << 20, (1 << 20) - 15, (1 << 20) - 16])
@pytest.mark.parametrize("cols", [16, 32, 33])
def test_the_most_rows(rows, cols):
    """2^20 rows, and the first and last counts on either side of 65535 blocks of sixteen: what comes back equals the rows of a small tensor that
    they repeat, and nothing behind is written."""
    base = _normal(4096, cols, cols)
    v = base.repeat(256, 1)[:rows].contiguous()

    def there_and_back(t, count, size, to, back):
        parts = [_bytes(f(count, cols)) for f in size]
        to(t, count, cols, parts[0][0], parts[1][0])
        out = torch.full((count * cols + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
        back(parts[0][0], parts[1][0], count, cols, out)
        torch.cuda.synchronize()
        assert all(bool((g == GUARD).all()) for _, g in parts) and bool((out[count * cols:] == -7.0).all())
        return out[:count * cols].reshape(count, cols), parts[0][0]

    for size, to, back in (((lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes), lords.lords_mxfp4_quantize, lords.lords_mxfp4_dequantize),
                           ((lords.lords_checkpoint_bytes, lords.lords_checkpoint_scales_bytes), lords.lords_checkpoint_store, lords.lords_checkpoint_load)):
        want, want_q = there_and_back(base, 4096, size, to, back)
        got, got_q = there_and_back(v, rows, size, to, back)
        assert torch.equal(got, want.repeat(256, 1)[:rows])
        assert torch.equal(got_q, want_q.repeat(256)[:got_q.numel()])


@pytest.mark.parametrize("M,n", [(17, 256), (33, 256), (64, 256), (20, 500), (32, 512)])
def test_a_call_of_one_launch_needs_no_workspace(M, n):
    """Few columns: x is converted inside the product's launch, so a workspace that would not hold it is no reason to refuse."""
    m = 384
    x, w = _normal(M, n, 1), _normal(m, n, 2)
    xq, wq = _four(M, n), _four(m, n)
    lords.lords_mxfp4_quantize(x, M, n, *xq)
    lords.lords_mxfp4_quantize(w, m, n, *wq)
    want = torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, want, f32=True)
    torch.cuda.synchronize()
    lords.lords_shutdown()
    try:
        lords.lords_init(0, 1024)
        y = torch.empty(M, m, device="cuda")
        lords.lords_mxfp4_forward(x, *wq, M, m, n, y, f32=True)
        assert lords.lords_last_launch_count() == 1 and torch.equal(y, want)
        # two launches, and no room for x between them: refused before anything is written
        wide = 12000
        a, b, out = _normal(M, wide, 3), _normal(m, wide, 4), torch.full((M, m), -7.0, device="cuda")
        bq = _four(m, wide)
        lords.lords_mxfp4_quantize(b, m, wide, *bq)
        with pytest.raises(lords.LordsError) as e:
            lords.lords_mxfp4_forward(a, *bq, M, m, wide, out, f32=True)
        torch.cuda.synchronize()
        assert e.value.status == -9 and bool((out == -7.0).all())
    finally:
        lords.lords_shutdown()
        lords.lords_init(0, 0)


# One row tile.  256 columns are one step: one launch up to 64 tokens.  12000 columns are 47 steps, six a CTA of eight: one launch up to four tokens, and
# up to ten (64 tokens x steps a CTA).
@pytest.mark.parametrize("m,n,M,launches", [(100, 256, 1, 1), (100, 256, 5, 1), (100, 256, 16, 1), (100, 256, 32, 1), (100, 256, 64, 1), (100, 256, 65, 2), (70, 12000, 1, 1),
                                            (70, 12000, 4, 1), (70, 12000, 10, 1), (70, 12000, 11, 2), (70, 12000, 16, 2), (70, 12000, 33, 2), (70, 12000, 64, 2)])
def test_launches_of_a_layer(m, n, M, launches):
    x, w = _normal(M, n, 1), _normal(m, n, 2)
    xq, wq = _four(M, n), _four(m, n)
    lords.lords_mxfp4_quantize(x, M, n, *xq)
    lords.lords_mxfp4_quantize(w, m, n, *wq)
    a, b = torch.empty(M, m, device="cuda"), torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, a, f32=True)
    lords.lords_mxfp4_forward(x, *wq, M, m, n, b, f32=True)
    assert lords.lords_last_launch_count() == launches
    assert torch.equal(a, b)


FIRST = """
import threading
import torch
from paper_2601_22716_b200 import binding as lords
M, m, n = {M}, 640, {n}
lords.lords_init(0, 0)
gen = torch.Generator(device="cuda").manual_seed(1)
four = lambda r, c: [torch.empty(f(r, c), dtype=torch.uint8, device="cuda") for f in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes)]
x, w = (torch.randn(r, n, generator=gen, device="cuda").to(torch.bfloat16) for r in (M, m))
xq, wq = four(M, n), four(m, n)
lords.lords_mxfp4_quantize(x, M, n, *xq)
lords.lords_mxfp4_quantize(w, m, n, *wq)
count = 8
streams, ys = [torch.cuda.Stream() for _ in range(count)], [torch.empty(M, m, device="cuda") for _ in range(count)]
torch.cuda.synchronize()
gate, bad = threading.Barrier(count), []

def work(k):
    torch.cuda.set_device(0)
    gate.wait()
    try:
        if M <= 4 and k % 2:         # (no scratch memory: calls on several streams do not meet)
            lords.lords_mxfp4_forward(x, *wq, M, m, n, ys[k], stream=streams[k], f32=True)
        else:
            lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, ys[k], stream=streams[k], f32=True)
    except Exception as e:
        bad.append(e)

threads = [threading.Thread(target=work, args=(k,)) for k in range(count)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
want = torch.empty(M, m, device="cuda")
lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, want, f32=True)
torch.cuda.synchronize()
assert not bad, bad
assert lords.lords_poll_status() == 0
assert all(torch.equal(y, want) for y in ys), [torch.equal(y, want) for y in ys]
"""


@pytest.mark.parametrize("M,n", [(3, 256), (3, 4096), (30, 256), (30, 4096), (100, 4096)])
def test_first_calls_from_several_threads(M, n):
    """How many clusters of a kernel fit is asked once; a thread that asks meanwhile gets the same answer."""
    subprocess.run([sys.executable, "-c", FIRST.format(M=M, n=n)], check=True, timeout=300)
