"""4-bit products on each kernel and tile, random shapes, sizes past 32 bits, and captured calls that share the workspace.

References are products in 64 bits of the operands' values as lords_mxfp4_dequantize gives them (tests/test_gpu_mx.py holds that call and the
quantisation to the definition)."""
import random

import pytest
import torch

from paper_2601_22716_b200 import binding as lords

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    lords.lords_init(0, 0)
    yield
    lords.lords_set_option("path", "auto")
    lords.lords_set_option("bn", "0")
    torch.cuda.synchronize()
    assert lords.lords_poll_status() == 0
    lords.lords_shutdown()


def _four(rows, cols):
    return [torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes)]


def _operand(rows, cols, seed, gain=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    v = (torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda")) * gain).to(torch.bfloat16)
    q = _four(rows, cols)
    lords.lords_mxfp4_quantize(v, rows, cols, *q)
    back = torch.empty_like(v)
    lords.lords_mxfp4_dequantize(*q, rows, cols, back)
    return v, q, back.double()


# as in tests/test_gpu_mx.py: fp32 sums, an addition per 64 columns and those that join the parts, each off by a unit of the largest possible sum
def _close(y, xv, wv):
    n = xv.shape[1]
    bound = (-(-n // 64) + 8) * (2.0**-23 * (xv.abs() @ wv.abs().T) + 2.0**-126)
    return bool(((y.double() - xv @ wv.T).abs() <= bound).all())


def _check(M, m, n, seed):
    _, xq, xv = _operand(M, n, seed)
    _, wq, wv = _operand(m, n, seed + 1, 0.05)
    y32 = torch.full((M, m), float("nan"), device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y32, f32=True)
    assert _close(y32, xv, wv), (M, m, n)
    y = torch.full((M * m + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y)
    assert torch.equal(y[:M * m].reshape(M, m), y32.to(torch.bfloat16)) and bool((y[M * m:] == -7.0).all())


@pytest.mark.parametrize("path,bn,name", [("decode", 0, "mxfp4_stream"), ("pair", 128, "mxfp4_pair"), ("pair", 256, "mxfp4_pair")])
@pytest.mark.parametrize("M,m,n", [(1, 1, 1), (3, 200, 70), (16, 384, 2048), (40, 257, 300), (100, 130, 5000), (128, 128, 257), (129, 513, 96), (255, 255, 255),
                                   (257, 300, 512), (600, 1100, 768), (2100, 640, 33)])
def test_every_kernel_takes_every_shape(path, bn, name, M, m, n):
    lords.lords_set_option("path", path)
    lords.lords_set_option("bn", str(bn))
    try:
        _check(M, m, n, M + m + n)
        assert lords.lords_last_path() == name
    finally:
        lords.lords_set_option("path", "auto")
        lords.lords_set_option("bn", "0")


def test_random_shapes():
    rng = random.Random(7)
    for k in range(60):
        M, m, n = (int(2 ** rng.uniform(0, top)) for top in (11, 12, 12))
        if rng.random() < 0.5:
            m, n = max(8, m // 8 * 8), max(32, n // 32 * 32)
        _check(M, m, n, 1000 + k)
    assert lords.lords_poll_status() == 0


def test_many_more_tiles_than_pairs():
    """Each pair runs a dozen tiles: accumulators, scales and the tiles on their way out are taken by turns."""
    _check(3000, 9000, 300, 5)
    _check(5000, 4000, 1000, 6)


def test_a_layer_s_token_counts_agree():
    """The layer's call, whichever way it takes x, has the bits of the two calls it stands for, at every count around its borders."""
    m, n = 640, 2048
    _, wq, _ = _operand(m, n, 3, 0.05)
    x, _, _ = _operand(160, n, 4)
    for M in (1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 160):
        xq = _four(M, n)
        lords.lords_mxfp4_quantize(x, M, n, *xq)
        a, b = torch.empty(M, m, device="cuda"), torch.empty(M, m, device="cuda")
        lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, a, f32=True)
        lords.lords_mxfp4_forward(x, *wq, M, m, n, b, f32=True)
        assert torch.equal(a, b), M


def test_clusters_of_several_streams_share_the_sms():
    """Calls of four token counts at once, each a cluster's: CTAs of different tiles lie on the same SMs and use their tensor memory together."""
    m, n = 1024, 4096
    counts = (1, 16, 64, 128)
    _, wq, _ = _operand(m, n, 5, 0.05)
    args, want = [], []
    for k, M in enumerate(counts):
        x, xq, _ = _operand(M, n, 20 + k)
        args.append((x, *wq) if M == 1 else (*xq, *wq))
        want.append(torch.empty(M, m, device="cuda"))
    calls = [lords.lords_mxfp4_forward if M == 1 else lords.lords_mxfp4_matmul for M in counts]
    for f, a, M, y in zip(calls, args, counts, want):
        f(*a, M, m, n, y, f32=True)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in counts]
    got = [[torch.empty_like(y) for _ in range(50)] for y in want]
    torch.cuda.synchronize()
    for r in range(50):
        for k, M in enumerate(counts):
            calls[k](*args[k], M, m, n, got[k][r], stream=streams[k], f32=True)
    torch.cuda.synchronize()
    assert lords.lords_poll_status() == 0
    assert all(torch.equal(y, want[k]) for k in range(len(counts)) for y in got[k])


@pytest.mark.parametrize("captured", [False, True])
def test_weights_written_right_before_the_layer(captured):
    """Neither of the layer's launches reads W before what came ahead of them has ended, a copy and the quantisation of the new weights included."""
    m, n = 4096, 4096
    gen = torch.Generator(device="cuda").manual_seed(11)
    ws = [(torch.randn(m, n, generator=gen, device="cuda") * 0.05).to(torch.bfloat16) for _ in range(3)]
    four, w = _four(m, n), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    for M in (8, 24, 64, 100):
        x = torch.randn(M, n, generator=gen, device="cuda").to(torch.bfloat16)
        want = []
        for v in ws:
            q, y = _four(m, n), torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
            lords.lords_mxfp4_quantize(v, m, n, *q)
            torch.cuda.synchronize()
            lords.lords_mxfp4_forward(x, *q, M, m, n, y)
            torch.cuda.synchronize()
            want.append(y)
        got = [torch.empty(M, m, dtype=torch.bfloat16, device="cuda") for _ in range(12)]
        stream = torch.cuda.Stream()

        def chain():
            for k, y in enumerate(got):
                if k % 2:
                    w.copy_(ws[k % 3])
                    lords.lords_mxfp4_quantize(w, m, n, *four)
                else:
                    lords.lords_mxfp4_quantize(ws[k % 3], m, n, *four)
                lords.lords_mxfp4_forward(x, *four, M, m, n, y)

        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    chain()
            for _ in range(10):
                for y in got:
                    y.zero_()
                graph.replay() if captured else chain()
                torch.cuda.synchronize()
                for k, y in enumerate(got):
                    assert torch.equal(y, want[k % 3]), (M, k)


@pytest.mark.parametrize("m,n", [(129, 40), (300, 256), (640, 700), (260, 1000), (1000, 2731), (4096, 4096), (5000, 513), (70, 12000), (20000, 256)])
def test_a_layer_on_one_launch_or_two(m, n):
    """Few steps a CTA: x is converted inside the product's launch up to 64 tokens x steps, by a launch of its own above; both have the same bits."""
    wide = (n + 7) // 8 * 8
    _, wq, _ = _operand(m, n, 3, 0.05)
    x, _, _ = _operand(72, wide, 4)
    x = x[:, :n].contiguous()
    launches = set()
    for M in (5, 6, 8, 10, 12, 13, 16, 17, 20, 21, 22, 31, 32, 33, 40, 63, 64, 65, 72):
        xq = _four(M, n)
        lords.lords_mxfp4_quantize(x, M, n, *xq)
        a, b = torch.empty(M, m, dtype=torch.bfloat16, device="cuda"), torch.full((M * m + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
        lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, a)
        lords.lords_mxfp4_forward(x, *wq, M, m, n, b)
        launches.add(lords.lords_last_launch_count())
        assert torch.equal(a, b[:M * m].reshape(M, m)) and bool((b[M * m:] == -7.0).all()), M
    assert launches <= {1, 2}


@pytest.mark.parametrize("cols", [33, 34, 35, 36, 37, 38, 39, 41, 63, 95, 127, 129, 131, 250, 517, 1023])
def test_rows_that_begin_anywhere(cols):
    """Row i of a width of 8 k + d begins d i values behind a 16-byte boundary, and the last one ends inside a word: what is read equals the same
    rows of a tensor whose width leaves them aligned, the values behind them zero."""
    wide = (cols + 31) // 32 * 32
    for rows in (1, 2, 5, 8, 9, 70):
        gen = torch.Generator(device="cuda").manual_seed(rows * 4096 + cols)
        v = torch.randn(rows, cols, generator=gen, device="cuda").to(torch.bfloat16)
        room = torch.full((rows * cols + 16,), float("inf"), dtype=torch.bfloat16, device="cuda")       # what lies behind belongs to nothing
        room[:rows * cols] = v.reshape(-1)
        odd, even = room[:rows * cols], torch.zeros(rows, wide, dtype=torch.bfloat16, device="cuda")
        even[:, :cols] = v
        a, at, b, bt = _four(rows, cols), _four(cols, rows), _four(rows, wide), _four(wide, rows)
        lords.lords_mxfp4_quantize(odd, rows, cols, *a, *at)
        lords.lords_mxfp4_quantize(even, rows, wide, *b, *bt)
        assert all(torch.equal(x, y) for x, y in zip(a, b)), rows
        pitch = lords.lords_mxfp4_codes_bytes(1, rows)
        assert torch.equal(at[0], bt[0][:cols * pitch]), rows
        size = lords.lords_checkpoint_bytes(rows, cols), lords.lords_checkpoint_scales_bytes(rows, cols)
        assert size == (lords.lords_checkpoint_bytes(rows, wide), lords.lords_checkpoint_scales_bytes(rows, wide))
        one, two = ([torch.zeros(k, dtype=torch.uint8, device="cuda") for k in size] for _ in range(2))
        lords.lords_checkpoint_store(odd, rows, cols, *one)
        lords.lords_checkpoint_store(even, rows, wide, *two)
        assert all(torch.equal(x, y) for x, y in zip(one, two)), rows
        _, wq, _ = _operand(40, cols, 9)
        y, z = torch.empty(rows, 40, device="cuda"), torch.empty(rows, 40, device="cuda")
        lords.lords_mxfp4_matmul(*a, *wq, rows, 40, cols, y, f32=True)
        lords.lords_mxfp4_forward(odd, *wq, rows, 40, cols, z, f32=True)
        assert torch.equal(y, z), rows


def test_sizes_past_32_bits():
    """More than 2^31 values, more than 2^32 bytes: the last rows and columns of every call."""
    rows, cols = 140000, 16000                # 2.24e9 values, 4.5 GB
    v = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    tail = torch.randn(200, cols, generator=gen, device="cuda").to(torch.bfloat16)
    v[-200:] = tail
    q, qt = _four(rows, cols), _four(cols, rows)
    lords.lords_mxfp4_quantize(v, rows, cols, *q, *qt)
    small = _four(200, cols)
    lords.lords_mxfp4_quantize(tail.contiguous(), 200, cols, *small)
    pitch = -(-cols // 32) * 16
    assert torch.equal(q[0][-200 * pitch:], small[0]) and not bool(q[0][: 1000 * pitch].any())
    # along the columns: rows - 200 is a multiple of neither 32 nor 128, so compare the values
    back = torch.empty(cols, rows, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_dequantize(*qt, cols, rows, back)
    first = (rows - 200) // 32 * 32
    block = torch.zeros(cols, rows - first, dtype=torch.bfloat16, device="cuda")
    block[:, rows - 200 - first:] = tail.T
    bq = _four(cols, rows - first)
    lords.lords_mxfp4_quantize(block, cols, rows - first, *bq)
    want = torch.empty_like(block)
    lords.lords_mxfp4_dequantize(*bq, cols, rows - first, want)
    assert torch.equal(back[:, first:], want) and not bool(back[:, :1000].any())
    del back, block
    e = torch.empty(lords.lords_checkpoint_scales_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    c = torch.empty(lords.lords_checkpoint_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    lords.lords_checkpoint_store(v, rows, cols, c, e)
    out = torch.empty_like(v)
    lords.lords_checkpoint_load(c, e, rows, cols, out)
    assert bool(((out[-200:].double() - tail.double()).abs() <= 2.0**-7 * tail.double().abs().amax(1, keepdim=True)).all()) and not bool(out[:1000].any())
    del out, c, e, qt
    # a product whose result has more than 2^31 values
    w = _operand(cols, 96, 9)
    x = torch.zeros(rows, 96, dtype=torch.bfloat16, device="cuda")
    x[-300:] = torch.randn(300, 96, generator=gen, device="cuda").to(torch.bfloat16)
    xq = _four(rows, 96)
    lords.lords_mxfp4_quantize(x, rows, 96, *xq)
    xv = torch.empty_like(x)
    lords.lords_mxfp4_dequantize(*xq, rows, 96, xv)
    y = v                                     # its buffer
    lords.lords_mxfp4_matmul(*xq, *w[1], rows, cols, 96, y)
    want = xv[-300:].double() @ w[2].T
    assert bool(((y[-300:].double() - want).abs() <= 2.0**-8 * want.abs() + 1e-5 * want.abs().amax()).all()) and not bool(y[:1000].any())


def test_two_captured_graphs_share_the_workspace():
    """x in 4 bits and a checkpoint's values lie in the library's workspace: graphs replayed by turns on one stream, and eager calls between."""
    m, n = 512, 1024
    sets = []
    for k, M in enumerate((48, 300)):
        x, _, _ = _operand(M, n, 50 + k)
        _, wq, _ = _operand(m, n, 60 + k, 0.05)
        y = torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
        lords.lords_mxfp4_forward(x, *wq, M, m, n, y)
        torch.cuda.synchronize()
        sets.append((x, wq, M, y, y.clone()))
    graphs = []
    for x, wq, M, y, _ in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lords.lords_mxfp4_forward(x, *wq, M, m, n, y)
        graphs.append(g)
    for turn in range(6):
        for (x, wq, M, y, want), g in zip(sets, graphs):
            y.fill_(-1)
            g.replay()
            if turn % 2:
                z = torch.empty_like(y)
                lords.lords_mxfp4_forward(x, *wq, M, m, n, z)
                assert torch.equal(z, want)
            assert torch.equal(y, want)


def test_calls_from_two_threads():
    """Host threads with a stream each, on calls without scratch memory."""
    import threading
    m, n, M = 256, 2048, 3
    x, xq, _ = _operand(M, n, 1)
    _, wq, _ = _operand(m, n, 2, 0.05)
    want = torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_forward(x, *wq, M, m, n, want, f32=True)
    torch.cuda.synchronize()
    bad = []

    def work():
        s = torch.cuda.Stream()
        ys = [torch.empty(M, m, device="cuda") for _ in range(50)]
        torch.cuda.synchronize()
        for k, y in enumerate(ys):
            if k % 2:
                lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y, stream=s, f32=True)
            else:
                lords.lords_mxfp4_forward(x, *wq, M, m, n, y, stream=s, f32=True)
        s.synchronize()
        if not all(torch.equal(y, want) for y in ys):
            bad.append(1)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_a_small_workspace_is_gone_through_in_parts():
    m, n, M = 384, 2048, 1500
    x, xq, _ = _operand(M, n, 1)
    _, wq, _ = _operand(m, n, 2, 0.05)
    want, want32 = torch.empty(M, m, dtype=torch.bfloat16, device="cuda"), torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, want)
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, want32, f32=True)
    torch.cuda.synchronize()
    lords.lords_shutdown()
    try:
        for room in (1 << 20, 300 << 10, 150 << 10):
            lords.lords_init(0, room)
            for dtype, ref in ((torch.bfloat16, want), (torch.float32, want32)):
                y = torch.full((M * m + 64,), -7.0, dtype=dtype, device="cuda")
                lords.lords_mxfp4_forward(x, *wq, M, m, n, y, f32=dtype == torch.float32)
                assert torch.equal(y[:M * m].reshape(M, m), ref) and bool((y[M * m:] == -7.0).all())
            assert lords.lords_poll_status() == 0
        lords.lords_init(0, 100 << 10)          # 128 tokens take 136 KiB
        with pytest.raises(lords.LordsError) as e:
            lords.lords_mxfp4_forward(x, *wq, M, m, n, want)
        assert e.value.status == -9
    finally:
        lords.lords_shutdown()
        lords.lords_init(0, 0)


def _at16(t):
    """The same values 16 bytes into a buffer that begins at a multiple of 32."""
    whole = torch.empty(t.numel() * t.element_size() + 48, dtype=torch.uint8, device="cuda")
    part = whole[16:16 + t.numel() * t.element_size()].view(t.dtype).reshape(t.shape)
    part.copy_(t)
    assert part.data_ptr() % 32 == 16
    return part


@pytest.mark.parametrize("M,m,n", [(3, 256, 512), (40, 256, 512), (300, 512, 1024)])
def test_addresses_at_odd_multiples_of_16(M, m, n):
    x, xq, _ = _operand(M, n, 1)
    w, wq, _ = _operand(m, n, 2, 0.05)
    want = torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, want)
    x16, w16 = _at16(x), _at16(w)
    qs = [_at16(q) for q in (*_four(m, n), *_four(n, m))]
    lords.lords_mxfp4_quantize(w16, m, n, *qs)
    ref = [*_four(m, n), *_four(n, m)]
    lords.lords_mxfp4_quantize(w, m, n, *ref)
    assert all(torch.equal(a, b) for a, b in zip(qs, ref))
    y = _at16(torch.empty_like(want))
    lords.lords_mxfp4_forward(x16, qs[0], qs[1], M, m, n, y)
    assert torch.equal(y, want)
    y.zero_()
    lords.lords_mxfp4_matmul(*[_at16(q) for q in xq], qs[0], qs[1], M, m, n, y)
    assert torch.equal(y, want)
    back, back16 = torch.empty_like(w), _at16(torch.empty_like(w))
    lords.lords_mxfp4_dequantize(*wq, m, n, back)
    lords.lords_mxfp4_dequantize(*[_at16(q) for q in wq], m, n, back16)
    assert torch.equal(back, back16)
    def kept(v, at):
        q = at(torch.empty(lords.lords_checkpoint_bytes(M, n), dtype=torch.uint8, device="cuda"))
        e = at(torch.empty(lords.lords_checkpoint_scales_bytes(M, n), dtype=torch.uint8, device="cuda"))
        out = at(torch.empty_like(v))
        lords.lords_checkpoint_store(v, M, n, q, e)
        lords.lords_checkpoint_load(q, e, M, n, out)
        return q, e, out
    assert all(torch.equal(a, b) for a, b in zip(kept(x, lambda t: t), kept(x16, _at16)))


def test_sizes_that_no_int_holds_are_refused():
    x, xq, _ = _operand(4, 64, 1)
    y = torch.empty(4, 4, dtype=torch.bfloat16, device="cuda")
    for bad in (2**32 + 4, 2**70, -2**40):
        with pytest.raises(lords.LordsError) as e:
            lords.lords_mxfp4_matmul(*xq, *xq, bad, 4, 64, y)
        assert e.value.status == -2
        with pytest.raises(lords.LordsError) as e:
            lords.lords_mxfp4_quantize(x, 4, bad, *xq)
        assert e.value.status == -2
