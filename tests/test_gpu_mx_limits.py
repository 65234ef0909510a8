"""Microscaled formats at the ends of their ranges."""
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
