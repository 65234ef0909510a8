"""Microscaled formats on the GPU against the definition in 64 bits (oracle/mx.py)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import mx
from paper_2601_22716_b200 import binding as lords
from paper_2601_22716_b200 import inputs

pytestmark = pytest.mark.gpu

GUARD = 0xA5


@pytest.fixture(scope="module", autouse=True)
def _lib():
    lords.lords_init(0, 0)
    yield
    torch.cuda.synchronize()
    assert lords.lords_poll_status() == 0
    lords.lords_shutdown()


def _bytes(count):
    """A buffer of `count` bytes with a guard behind it."""
    whole = torch.full((count + 256,), GUARD, dtype=torch.uint8, device="cuda")
    return whole[:count], whole[count:]


def _untouched(*guards):
    return all(bool((g == GUARD).all()) for g in guards)


def _values(rows, cols, seed, special=False):
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(rows, cols, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen))
    if special:      # an empty row, subnormal and huge ones, blocks that are not finite, exact ties
        flat = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
        for i, edit in enumerate((lambda r: r * 0, lambda r: r * 2.0**-130, lambda r: r.sign() * 3e38, lambda r: flat.repeat(cols // 8 + 1)[:cols] * r.sign())):
            if i < rows:
                v[i] = edit(v[i])
        if rows > 5:
            v[4, cols // 2] = float("inf")
            v[5, cols - 1] = float("nan")
    return v.to(torch.bfloat16)


def _quantize(v, along=True, across=False):
    rows, cols = v.shape
    bufs, guards = [], []
    for wanted, (r, c) in ((along, (rows, cols)), (across, (cols, rows))):
        for size in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes):
            b, g = _bytes(size(r, c)) if wanted else (None, None)
            bufs.append(b)
            guards += [g] if wanted else []
    lords.lords_mxfp4_quantize(v, rows, cols, *bufs)
    assert _untouched(*guards)
    return bufs


def _oracle4(v):
    codes, E = mx.quantize4(v.double().cpu().numpy())
    return codes, E, mx.values4(codes, E)


SHAPES = [(1, 1), (1, 31), (1, 4096), (3, 33), (5, 8), (31, 32), (32, 127), (33, 128), (64, 250), (127, 129), (128, 128), (129, 1000), (130, 257), (260, 2731), (2048, 40)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_four_bits_are_the_definition_s(rows, cols):
    v = _values(rows, cols, rows * 7 + cols, special=True)
    codes, E, ref = _oracle4(v)
    want = mx.pack4(codes, E)
    tcodes, tE, _ = _oracle4(v.T)
    want_t = mx.pack4(tcodes, tE)
    d = v.cuda()
    for along, across in ((True, False), (False, True), (True, True)):
        got = _quantize(d, along, across)
        for k, w in enumerate((*want, *want_t)):
            if got[k] is not None:
                assert np.array_equal(got[k].cpu().numpy(), w), (along, across, k)
    got = _quantize(d)
    whole = torch.full((rows * cols + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_dequantize(got[0], got[1], rows, cols, whole)
    assert np.array_equal(whole[:rows * cols].double().cpu().numpy(), ref.reshape(-1), equal_nan=True)
    assert bool((whole[rows * cols:] == -7.0).all())


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_eight_bits_are_the_definition_s(rows, cols):
    v = _values(rows, cols, rows * 11 + cols, special=True)
    q, E = mx.quantize8(v.double().numpy())
    want_q, want_e = mx.pack8(q, E)
    (dq, gq), (de, ge) = _bytes(lords.lords_checkpoint_bytes(rows, cols)), _bytes(lords.lords_checkpoint_scales_bytes(rows, cols))
    lords.lords_checkpoint_store(v.cuda(), rows, cols, dq, de)
    assert np.array_equal(dq.cpu().numpy(), want_q) and np.array_equal(de.cpu().numpy(), want_e) and _untouched(gq, ge)
    whole = torch.full((rows * cols + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
    lords.lords_checkpoint_load(dq, de, rows, cols, whole)
    assert np.array_equal(whole[:rows * cols].double().cpu().numpy(), mx.values8(q, E).reshape(-1), equal_nan=True)
    assert bool((whole[rows * cols:] == -7.0).all())


def test_every_scale_and_code_of_the_formats_is_read_back():
    """All 253 scales that a bf16 block can get, and not-a-number, with all values."""
    rows = 254
    E = np.arange(-127, 127)[:, None].copy()
    E[253] = 128
    codes = np.tile(np.arange(32, dtype=np.uint8) % 16, (rows, 1))
    out = torch.empty(rows, 32, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_dequantize(*[torch.from_numpy(b).cuda() for b in mx.pack4(codes, E)], rows, 32, out)
    assert np.array_equal(out.double().cpu().numpy(), mx.values4(codes, E), equal_nan=True)
    E = np.arange(-127, 129)[:, None].copy()
    q = np.tile(np.arange(-127, 128, 8, dtype=np.int8), (256, 1))
    out = torch.empty(256, 32, dtype=torch.bfloat16, device="cuda")
    lords.lords_checkpoint_load(*[torch.from_numpy(b).cuda() for b in mx.pack8(q, E)], 256, 32, out)
    assert np.array_equal(out.double().cpu().numpy(), mx.values8(q, E), equal_nan=True)


# ---- the product -------------------------------------------------------------------------------------------------
# Operands are exact.  Sums are fp32: an MMA adds 64 products to the sum so far and cuts what does not fit 24 bits off, so each of the
# ceil(n / 64) additions (and of the at most eight that join the parts of a sum) is off by at most a unit of the largest magnitude that the
# sum can have, the sum of the products' magnitudes.  A sum below 2^-126, where fp32's normal numbers end, may become zero at any of them
# (2^-100 times 2^-60 does).
def _bound(xv, wv, n):
    adds = -(-n // 64) + 8
    return adds * (2.0**-23 * (np.abs(xv) @ np.abs(wv).T) + 2.0**-126)


def _rounded(y32):
    return y32.to(torch.bfloat16)


PRODUCTS = [(1, 1, 1), (1, 128, 32), (1, 130, 96), (2, 127, 64), (3, 300, 2731), (8, 256, 256), (15, 129, 257), (16, 1000, 8192), (17, 256, 33), (31, 100, 1000),
            (33, 500, 640), (64, 384, 4096), (65, 129, 511), (96, 1024, 1024), (128, 256, 2048), (129, 640, 288), (200, 1000, 2731), (256, 2048, 512),
            (300, 700, 1500), (513, 1300, 1030), (1024, 512, 96), (2048, 4096, 128)]


@pytest.mark.parametrize("M,m,n", PRODUCTS)
def test_product(M, m, n):
    x, w = _values(M, n, M + 3 * n).cuda(), (_values(m, n, m + 5 * n) * 0.05).cuda()
    xq, wq = _quantize(x)[:2], _quantize(w)[:2]
    xv, wv = _oracle4(x)[2], _oracle4(w)[2]
    whole = torch.full((M * m + 64,), float("nan"), device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, whole, f32=True)
    y32 = whole[:M * m].reshape(M, m)
    assert bool(torch.isnan(whole[M * m:]).all())
    err = np.abs(y32.double().cpu().numpy() - xv @ wv.T)
    assert (err <= _bound(xv, wv, n)).all(), float((err / np.maximum(_bound(xv, wv, n), 1e-300)).max())
    y = torch.full((M * m + 64,), -7.0, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y)
    assert torch.equal(y[:M * m].reshape(M, m), _rounded(y32)) and bool((y[M * m:] == -7.0).all())
    # the layer's call brings x to 4 bits by itself: the same to the last bit
    z = torch.full((M, m), float("nan"), device="cuda")
    lords.lords_mxfp4_forward(x, *wq, M, m, n, z, f32=True)
    assert torch.equal(z, y32)
    zb = torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_forward(x, *wq, M, m, n, zb)
    assert torch.equal(zb, _rounded(y32))
    assert lords.lords_poll_status() == 0


@pytest.mark.parametrize("M,m,n", [(4, 256, 300), (40, 256, 300), (300, 520, 300)])
def test_wide_ranges_and_blocks_that_are_not_numbers(M, m, n):
    x, w = _values(M, n, 1, special=False), _values(m, n, 2)
    x[0] *= 2.0**60
    x[1] *= 2.0**-100
    w[3] *= 2.0**-60
    x[2, 40], w[5, 299], w[7, 0] = float("inf"), float("nan"), float("-inf")
    xq, wq = _quantize(x.cuda())[:2], _quantize(w.cuda())[:2]
    xv, wv = _oracle4(x)[2], _oracle4(w)[2]
    y = torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y, f32=True)
    got = y.double().cpu().numpy()
    nan = np.zeros((M, m), dtype=bool)
    nan[2], nan[:, 5], nan[:, 7] = True, True, True
    assert np.array_equal(np.isnan(got), nan)
    xz, wz = np.nan_to_num(xv), np.nan_to_num(wv)
    assert (np.abs(got - xz @ wz.T) <= _bound(xz, wz, n))[~nan].all()


def test_an_empty_operand_gives_zeros():
    M, m, n = 20, 130, 70
    x, w = torch.zeros(M, n, dtype=torch.bfloat16, device="cuda"), _values(m, n, 2).cuda()
    y = torch.full((M, m), 3.0, device="cuda")
    lords.lords_mxfp4_matmul(*_quantize(x)[:2], *_quantize(w)[:2], M, m, n, y, f32=True)
    assert bool((y == 0).all())


def test_runs_are_bit_identical():
    for M, m, n in ((16, 4096, 4096), (200, 1024, 8192), (1024, 1024, 2048)):
        x, w = _values(M, n, 1).cuda(), _values(m, n, 2).cuda()
        wq = _quantize(w)[:2]
        ys = [torch.empty(M, m, device="cuda") for _ in range(8)]
        for y in ys:
            lords.lords_mxfp4_forward(x, *wq, M, m, n, y, f32=True)
        assert all(torch.equal(y, ys[0]) for y in ys)


def test_results_follow_the_stream_s_order():
    """Weights, activations and results rewritten on the stream, with no wait between."""
    m, n = 512, 1024
    for M in (1, 16, 48, 512):
        xs = [_values(M, n, 10 + k).cuda() for k in range(6)]
        ws = [_values(m, n, 20 + k).cuda() for k in range(6)]
        want = []
        for x, w in zip(xs, ws):
            y = torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
            lords.lords_mxfp4_matmul(*_quantize(x)[:2], *_quantize(w)[:2], M, m, n, y)
            torch.cuda.synchronize()
            want.append(y)
        codes, scales, _, _ = _quantize(ws[0])
        x, y = xs[0].clone(), torch.empty(M, m, dtype=torch.bfloat16, device="cuda")
        got = []
        torch.cuda.synchronize()
        for k in range(6):
            x.copy_(xs[k])
            lords.lords_mxfp4_quantize(ws[k], m, n, codes, scales)
            lords.lords_mxfp4_forward(x, codes, scales, M, m, n, y)
            got.append(y.clone())
        assert all(torch.equal(a, b) for a, b in zip(got, want)), M


def test_other_streams_do_not_meet():
    """The product and the one-launch layer use no scratch memory: calls on two streams at once keep their results."""
    m, n = 1024, 4096
    for M, call in ((3, "forward"), (8, "matmul"), (256, "matmul")):
        args = []
        for k in range(2):
            x, w = _values(M, n, 30 + k).cuda(), _values(m, n, 40 + k).cuda()
            wq, xq = _quantize(w)[:2], _quantize(x)[:2]
            args.append((x, *wq) if call == "forward" else (*xq, *wq))
        fn = lords.lords_mxfp4_forward if call == "forward" else lords.lords_mxfp4_matmul
        want = [torch.empty(M, m, device="cuda") for _ in range(2)]
        for a, y in zip(args, want):
            fn(*a, M, m, n, y, f32=True)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        ys = [[torch.empty(M, m, device="cuda") for _ in range(20)] for _ in range(2)]
        torch.cuda.synchronize()
        for r in range(20):
            for k in range(2):
                fn(*args[k], M, m, n, ys[k][r], stream=streams[k], f32=True)
        torch.cuda.synchronize()
        assert all(torch.equal(y, want[k]) for k in range(2) for y in ys[k])


def test_a_captured_step_replays_on_new_inputs():
    M, m, n = 96, 384, 512
    x, w, g = (torch.empty(*s, dtype=torch.bfloat16, device="cuda") for s in ((M, n), (m, n), (M, m)))
    out = _step_buffers(M, m, n)
    for src, dst in ((_values(M, n, 1), x), (_values(m, n, 2), w), (_values(M, m, 3), g)):
        dst.copy_(src)
    _step(x, w, g, M, m, n, out)          # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(x, w, g, M, m, n, out)
    for seed in (5, 6):
        x.copy_(_values(M, n, seed))
        w.copy_(_values(m, n, seed + 10))
        g.copy_(_values(M, m, seed + 20))
        graph.replay()
        got = [t.clone() for t in out["results"]]
        _step(x, w, g, M, m, n, out)
        assert all(torch.equal(a, b) for a, b in zip(got, out["results"]))


# ---- a training step: the calls as they are used together ----------------------------------------------------------
def _step_buffers(M, m, n):
    def four(rows, cols):
        return [torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes)]
    return dict(x=four(M, n), xt=four(n, M), w=four(m, n), wt=four(n, m), g=four(M, m), gt=four(m, M),
                results=[torch.empty(M, m, device="cuda"), torch.empty(M, n, device="cuda"), torch.empty(m, n, device="cuda"), torch.empty(M, m, dtype=torch.bfloat16, device="cuda")])


def _step(x, w, g, M, m, n, b):
    y, dx, dW, yb = b["results"]
    lords.lords_mxfp4_quantize(x, M, n, *b["x"], *b["xt"])
    lords.lords_mxfp4_quantize(w, m, n, *b["w"], *b["wt"])
    lords.lords_mxfp4_matmul(*b["x"], *b["w"], M, m, n, y, f32=True)
    lords.lords_mxfp4_forward(x, *b["w"], M, m, n, yb)
    lords.lords_mxfp4_quantize(g, M, m, *b["g"], *b["gt"])
    lords.lords_mxfp4_matmul(*b["g"], *b["wt"], M, n, m, dx, f32=True)
    lords.lords_mxfp4_matmul(*b["gt"], *b["xt"], m, n, M, dW, f32=True)


@pytest.mark.parametrize("M,m,n", [(5, 64, 96), (37, 300, 257), (130, 520, 384), (512, 1024, 640)])
def test_training_step(M, m, n):
    x, w, g = _values(M, n, 1), _values(m, n, 2), _values(M, m, 3)
    g[M - 2:] = 0                         # padded tokens
    b = _step_buffers(M, m, n)
    _step(x.cuda(), w.cuda(), g.cuda(), M, m, n, b)
    y, dx, dW, yb = b["results"]
    for got, a, c in ((y, x, w), (dx, g, w.T), (dW, g.T, x.T)):
        av, cv = _oracle4(a)[2], _oracle4(c)[2]
        assert (np.abs(got.double().cpu().numpy() - av @ cv.T) <= _bound(av, cv, a.shape[1])).all()
    assert torch.equal(yb, _rounded(y))
    # differences: sum(g y) with the operands' 4-bit values is linear in every entry of W and x, so a step of 1 in one entry changes it by that
    # entry's gradient
    gv, xv = _oracle4(g.T)[2].T, _oracle4(x.T)[2].T
    loss = lambda W: float((gv * (xv @ W.T)).sum())  # noqa: E731
    W0 = w.double().numpy()
    for i, j in ((0, 0), (m // 2, n - 1), (m - 1, n // 3)):
        W1 = W0.copy()
        W1[i, j] += 1.0
        size = (np.abs(gv) * (np.abs(xv) @ np.abs(W1).T)).sum()          # what 64 bits round to
        assert abs(loss(W1) - loss(W0) - float(dW[i, j])) <= 1e-5 * (np.abs(gv[:, i]) @ np.abs(xv[:, j])) + 1e-12 * size


# ---- gradients from a checkpoint --------------------------------------------------------------------------------------
def _layer(m, n, r, M, bits, seed):
    lay = inputs.make_layer(m, n, r, M, bits=bits, seed=seed, scale_gain=0.1, scale_shift=0.05)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()  # noqa: E731
    q = torch.from_numpy(lords.lords_pack_codes(lay.codes, bits)).cuda()
    return lay, q, dev(lay.B), dev(lay.A)


GRADIENTS = [(64, 64, 4, 3, 4), (300, 258, 10, 37, 4), (256, 512, 32, 130, 3), (130, 200, 7, 65, 2), (1000, 2730, 16, 100, 4), (512, 1024, 128, 256, 4)]


@pytest.mark.parametrize("m,n,r,M,bits", GRADIENTS)
def test_gradients_from_a_checkpoint(m, n, r, M, bits):
    lay, q, B, A = _layer(m, n, r, M, bits, seed=m + n)
    x, g, W = _values(M, n, 1).cuda(), _values(M, m, 2).cuda(), (_values(m, n, 3) * 0.1).cuda()
    cq = torch.empty(lords.lords_checkpoint_bytes(M, n), dtype=torch.uint8, device="cuda")
    ce = torch.empty(lords.lords_checkpoint_scales_bytes(M, n), dtype=torch.uint8, device="cuda")
    lords.lords_checkpoint_store(x, M, n, cq, ce)
    xv = torch.empty_like(x)
    lords.lords_checkpoint_load(cq, ce, M, n, xv)
    new = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    cb = lay.codebook
    dB, dA, dB0, dA0 = new(m, r), new(r, n), new(m, r), new(r, n)
    lords.lords_linear_backward_factors_checkpoint(g, cq, ce, q, B, A, cb, bits, M, m, n, r, dB, dA)
    lords.lords_linear_backward_factors(g, xv, q, B, A, cb, bits, M, m, n, r, dB0, dA0)
    assert torch.equal(dB, dB0) and torch.equal(dA, dA0)
    # against the formula in 64 bits, from the oracle's own checkpoint: sums of m n M exact products in fp32 (1e-4 of the norm, as for the
    # gradients from bf16 activations)
    x64 = mx.values8(*mx.quantize8(x.double().cpu().numpy()))
    g64, B64, A64 = g.double().cpu().numpy(), mx.bf16_values(lay.B), mx.bf16_values(lay.A)
    G = g64.T @ x64
    level = cb.astype(np.float64)[lay.codes]
    near = lambda a, b: np.linalg.norm(a.double().cpu().numpy() - b) <= 1e-4 * np.linalg.norm(b)  # noqa: E731
    dS = G * level
    assert near(dB, dS @ A64.T) and near(dA, B64.T @ dS)
    # differences: the loss sum(g y) is linear in every entry of B
    loss = lambda Bm: float((g64 * (x64 @ (level * (Bm @ A64)).T)).sum())  # noqa: E731
    B1 = B64.copy()
    B1[m // 2, r - 1] += 1.0
    size = (np.abs(g64) * (np.abs(x64) @ (np.abs(level) * (np.abs(B1) @ np.abs(A64))).T)).sum()
    assert abs(loss(B1) - loss(B64) - float(dB[m // 2, r - 1])) <= 1e-4 * np.linalg.norm(dS @ A64.T) + 1e-12 * size
    dW, dW0 = new(m, n), new(m, n)
    for t in (dB, dA, dB0, dA0):
        t.fill_(float("nan"))
    lords.lords_linear_backward_qat_checkpoint(g, cq, ce, W, q, B, A, cb, bits, M, m, n, r, dW, dB, dA)
    lords.lords_linear_backward_qat(g, xv, W, q, B, A, cb, bits, M, m, n, r, dW0, dB0, dA0)
    assert torch.equal(dW, dW0) and torch.equal(dB, dB0) and torch.equal(dA, dA0)
    S = B64 @ A64
    dS = G * (level - W.double().cpu().numpy() / S)
    assert near(dW, G) and near(dB, dS @ A64.T) and near(dA, B64.T @ dS)
    # an output that is not asked for is not touched
    only = new(r, n)
    lords.lords_linear_backward_factors_checkpoint(g, cq, ce, q, B, A, cb, bits, M, m, n, r, None, only)
    assert torch.equal(only, dA0) or near(only, B64.T @ (G * level))
    assert oracle is not None and lords.lords_poll_status() == 0


def test_the_library_s_own_refusals():
    """Workspace too small for what a call keeps there; calls without scratch go through."""
    lords.lords_shutdown()
    lords.lords_init(0, 1 << 16)
    try:
        M, m, n, r, bits = 64, 256, 2048, 8, 4
        x, w = _values(M, n, 1).cuda(), _values(m, n, 2).cuda()
        wq, xq = _quantize(w)[:2], _quantize(x)[:2]
        y = torch.full((M, m), -7.0, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(lords.LordsError) as e:
            lords.lords_mxfp4_forward(x, *wq, M, m, n, y)
        assert e.value.status == -9
        lay, q, B, A = _layer(m, n, r, M, bits, 1)
        cq = torch.empty(lords.lords_checkpoint_bytes(M, n), dtype=torch.uint8, device="cuda")
        ce = torch.empty(lords.lords_checkpoint_scales_bytes(M, n), dtype=torch.uint8, device="cuda")
        lords.lords_checkpoint_store(x, M, n, cq, ce)
        dB, dA = torch.full((m, r), -7.0, device="cuda"), torch.full((r, n), -7.0, device="cuda")
        with pytest.raises(lords.LordsError) as e:
            lords.lords_linear_backward_factors_checkpoint(torch.zeros(M, m, dtype=torch.bfloat16, device="cuda"), cq, ce, q, B, A, lay.codebook, bits, M, m, n, r, dB, dA)
        assert e.value.status == -9
        torch.cuda.synchronize()
        assert bool((y == -7.0).all()) and bool((dB == -7.0).all()) and bool((dA == -7.0).all())
        lords.lords_mxfp4_matmul(*xq, *wq, M, m, n, y)
        lords.lords_mxfp4_forward(x, *wq, 4, m, n, y)
        torch.cuda.synchronize()
    finally:
        lords.lords_shutdown()
        lords.lords_init(0, 0)


@pytest.mark.parametrize("order", ["ascending", "shuffled", "with one large value"])
def test_every_bf16_pattern(order):
    """All 65536 patterns, subnormal numbers, infinities and NaNs among them, to both formats and back."""
    bits = np.arange(65536, dtype=np.uint16)
    if order == "shuffled":                     # nearly every block has a value that is not finite: those apart
        finite = bits[(bits & 0x7F80) != 0x7F80]
        bits = np.random.default_rng(1).permutation(finite)
    bits = bits[: len(bits) // 32 * 32].reshape(-1, 32).copy()
    if order == "with one large value":         # 1.0 first, so that the others are rounded on its grid
        bits[:, 0] = 0x3F80
    v = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16)
    v64 = mx.bf16_values(bits)
    rows, cols = bits.shape
    codes, E = mx.quantize4(v64)
    tcodes, tE = mx.quantize4(v64.T.copy())
    got = _quantize(v.cuda(), True, True)
    for g, w in zip(got, (*mx.pack4(codes, E), *mx.pack4(tcodes, tE))):
        assert np.array_equal(g.cpu().numpy(), w)
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    lords.lords_mxfp4_dequantize(got[0], got[1], rows, cols, out)
    assert np.array_equal(out.double().cpu().numpy(), mx.values4(codes, E), equal_nan=True)
    q, E8 = mx.quantize8(v64)
    dq, de = (torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (lords.lords_checkpoint_bytes, lords.lords_checkpoint_scales_bytes))
    lords.lords_checkpoint_store(v.cuda(), rows, cols, dq, de)
    for g, w in zip((dq, de), mx.pack8(q, E8)):
        assert np.array_equal(g.cpu().numpy(), w)
    lords.lords_checkpoint_load(dq, de, rows, cols, out)
    assert np.array_equal(out.double().cpu().numpy(), mx.values8(q, E8), equal_nan=True)
    # the same values on the way into a product: one row of identity weights after the other picks them out again
    eye = torch.eye(cols, dtype=torch.bfloat16, device="cuda")
    wq = _quantize(eye)[:2]
    x = v[:4].contiguous().cuda()
    y = torch.empty(4, cols, device="cuda")
    lords.lords_mxfp4_forward(x, *wq, 4, cols, cols, y, f32=True)
    want = mx.values4(codes[:4], E[:4])
    near = want * (np.abs(want) >= 2.0**-126)   # below fp32's normal numbers a sum may become zero
    got4 = y.double().cpu().numpy()
    assert np.array_equal(np.isnan(got4), np.isnan(want)) and ((got4 == want) | (got4 == near) | np.isnan(want)).all()


def test_with_the_low_rank_scaled_layers_on_one_stream():
    """A chain of layers of either kind, activations kept on the way and gradients taken, without a wait between."""
    M, h, r, bits = 24, 512, 8, 4
    lay, q, B, A = _layer(h, h, r, M, bits, 3)
    w = (_values(h, h, 4) * 0.02).to(torch.bfloat16).cuda()
    wq = _quantize(w)[:2]
    x0, g = _values(M, h, 5).cuda(), _values(M, h, 6).cuda()
    torch.cuda.synchronize()

    def chain(wait):
        done = torch.cuda.synchronize if wait else (lambda: None)
        out = []
        x = x0
        for _ in range(4):
            a = torch.empty(M, h, dtype=torch.bfloat16, device="cuda")
            lords.lords_linear_forward_bits(x, q, B, A, lay.codebook, bits, M, h, h, r, a)
            done()
            cq = torch.empty(lords.lords_checkpoint_bytes(M, h), dtype=torch.uint8, device="cuda")
            ce = torch.empty(lords.lords_checkpoint_scales_bytes(M, h), dtype=torch.uint8, device="cuda")
            lords.lords_checkpoint_store(a, M, h, cq, ce)
            done()
            b = torch.empty(M, h, dtype=torch.bfloat16, device="cuda")
            lords.lords_mxfp4_forward(a, *wq, M, h, h, b)
            done()
            dB, dA = torch.empty(h, r, device="cuda"), torch.empty(r, h, device="cuda")
            lords.lords_linear_backward_factors_checkpoint(g, cq, ce, q, B, A, lay.codebook, bits, M, h, h, r, dB, dA)
            done()
            x = b
            out += [a, b, dB, dA]
        torch.cuda.synchronize()
        return out

    want = chain(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(chain(False), want))
    assert lords.lords_poll_status() == 0


def test_a_status_that_a_kernel_left_is_reported_and_cleared():
    M, m, n = 20, 256, 512
    x, w = _values(M, n, 1).cuda(), _values(m, n, 2).cuda()
    wq = _quantize(w)[:2]
    y = torch.empty(M, m, device="cuda")
    lords.lords_mxfp4_forward(x, *wq, M, m, n, y, f32=True)
    want = y.clone()
    assert lords.lords_poll_status() == 0
    lords.lords_set_option("inject_status", "-8")
    for rows in (2, 20):
        lords.lords_mxfp4_forward(x, *wq, rows, m, n, y)
    assert lords.lords_poll_status() == -8
    lords.lords_mxfp4_forward(x, *wq, M, m, n, y, f32=True)
    assert lords.lords_poll_status() == 0 and torch.equal(y, want)


def test_the_first_call_of_a_process_may_be_captured():
    """Nothing that a capture forbids happens at a kernel's first call."""
    import subprocess
    import sys
    code = """
import torch
from paper_2601_22716_b200 import binding as lords
lords.lords_init(0, 0)
def four(rows, cols):
    return [torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (lords.lords_mxfp4_codes_bytes, lords.lords_mxfp4_scales_bytes)]
m, n = 512, 1024
w = torch.randn(m, n, device="cuda").to(torch.bfloat16)
for M in (1, 12, 48, 100, 700):
    x, y = torch.randn(M, n, device="cuda").to(torch.bfloat16), torch.zeros(M, m, device="cuda")
    q, back = four(m, n), torch.zeros_like(w)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lords.lords_mxfp4_quantize(w, m, n, *q)
        lords.lords_mxfp4_dequantize(*q, m, n, back)
        lords.lords_mxfp4_forward(x, *q, M, m, n, y, f32=True)
    g.replay()
    torch.cuda.synchronize()
    z = torch.empty_like(y)
    lords.lords_mxfp4_forward(x, *q, M, m, n, z, f32=True)
    assert lords.lords_poll_status() == 0 and torch.equal(y, z) and bool(back.any()) and bool(y.any())
"""
    subprocess.run([sys.executable, "-c", code], check=True)
