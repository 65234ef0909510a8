"""Gradients from a checkpoint whose values the workspace does not hold at once: the tokens go through it in parts."""
import numpy as np
import pytest
import torch

from paper_2601_22716_b200 import binding as lords
from paper_2601_22716_b200 import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    lords.lords_init(0, 0)
    yield
    torch.cuda.synchronize()
    assert lords.lords_poll_status() == 0
    lords.lords_shutdown()


class Step:
    """A layer, its latent weight, the gradient of y and the input's checkpoint; and what the gradients are in 64 bits."""

    def __init__(self, m, n, r, M, bits, seed):
        lay = inputs.make_layer(m, n, r, 1, bits=bits, seed=seed, scale_gain=0.1, scale_shift=0.5)
        self.sizes, self.cb, self.bits = (M, m, n, r), lay.codebook, bits
        self.q = torch.from_numpy(lords.lords_pack_codes(lay.codes, bits)).cuda()
        bf16 = lambda b: torch.from_numpy(b.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
        self.B, self.A = bf16(lay.B), bf16(lay.A)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        x = normal(M, n).to(torch.bfloat16)
        self.g, self.W = normal(M, m).to(torch.bfloat16), (normal(m, n) * 0.1).to(torch.bfloat16)
        self.cq = torch.empty(lords.lords_checkpoint_bytes(M, n), dtype=torch.uint8, device="cuda")
        self.ce = torch.empty(lords.lords_checkpoint_scales_bytes(M, n), dtype=torch.uint8, device="cuda")
        lords.lords_checkpoint_store(x, M, n, self.cq, self.ce)
        self.x = torch.empty_like(x)
        lords.lords_checkpoint_load(self.cq, self.ce, M, n, self.x)
        torch.cuda.synchronize()
        self.level = torch.from_numpy(np.ascontiguousarray(lay.codebook[lay.codes])).cuda().double()

    def exact(self, qat):
        """dW, dB, dA, and the sums of the magnitudes that they are sums of."""
        g, x, A, B = self.g.double(), self.x.double(), self.A.double(), self.B.double()
        G, size = g.T @ x, g.abs().T @ x.abs()
        factor = self.level - self.W.double() / (B @ A) if qat else self.level
        return (G, (G * factor) @ A.T, B.T @ (G * factor)), (size, (size * factor.abs()) @ A.abs().T, B.abs().T @ (size * factor.abs()))

    def run(self, qat, checkpoint, wanted=(True, True, True)):
        """dW (QAT only), dB, dA; those that are not wanted keep what they hold."""
        M, m, n, r = self.sizes
        out = [torch.full(s, -7.0, device="cuda") for s in ((m, n), (m, r), (r, n))]
        dW, dB, dA = (o if w else None for o, w in zip(out, wanted))
        x = (self.cq, self.ce) if checkpoint else (self.x,)
        tail = (self.q, self.B, self.A, self.cb, self.bits, M, m, n, r)
        if qat:
            f = lords.lords_linear_backward_qat_checkpoint if checkpoint else lords.lords_linear_backward_qat
            f(self.g, *x, self.W, *tail, dW, dB, dA)
        else:
            f = lords.lords_linear_backward_factors_checkpoint if checkpoint else lords.lords_linear_backward_factors
            f(self.g, *x, *tail, dB, dA)
        return out

    def check(self, got, qat):
        """Every value is a sum over tokens and then over columns or rows, in fp32 from exact products: at most M + m + n additions, each off by at
        most a unit of the largest magnitude that the sum can have.  (QAT's factor L - W / S has errors of its own: 1e-4 of the norm, as the
        gradients from bf16 activations are tested.)"""
        M, m, n, _ = self.sizes
        want, size = self.exact(qat)
        for k, (a, b, s) in enumerate(zip(got, want, size)):
            if k == 0 and not qat:
                continue
            if qat and k > 0:
                assert float((a.double() - b).norm()) <= 1e-4 * float(b.norm()), k
            else:
                assert bool(((a.double() - b).abs() <= (M + m + n) * 2.0**-23 * s).all()), k


@pytest.fixture
def workspace():
    def bind(room):
        torch.cuda.synchronize()
        lords.lords_shutdown()
        lords.lords_init(0, room)

    yield bind
    bind(0)


# Workspaces between what 64 tokens take and what all take; in the last of each the contributions of the tensor schedule do not fit as well.
@pytest.mark.parametrize("m,n,r,M,bits,rooms", [(256, 512, 8, 300, 4, (500 << 10, 300 << 10, 240 << 10, 70 << 10)),
                                                (384, 256, 12, 129, 4, (120 << 10, 90 << 10, 33 << 10)),
                                                (128, 1024, 32, 1000, 3, (1500 << 10, 900 << 10, 520 << 10, 140 << 10)),
                                                (300, 516, 20, 200, 2, (900 << 10, 700 << 10, 500 << 10, 70 << 10)),
                                                (200, 390, 5, 321, 4, (400 << 10, 250 << 10, 60 << 10))])
def test_gradients_in_parts(workspace, m, n, r, M, bits, rooms):
    s = Step(m, n, r, M, bits, m + n)
    whole = {qat: s.run(qat, True) for qat in (False, True)}
    for qat in (False, True):
        assert all(torch.equal(a, b) for a, b in zip(whole[qat], s.run(qat, False)))        # all at once: the values' own gradients, to the last bit
    more = 0
    for room in rooms:
        workspace(room)
        for qat in (False, True):
            got = s.run(qat, True)
            launches = lords.lords_last_launch_count()
            s.check(got, qat)
            again = s.run(qat, True)
            assert all(torch.equal(a, b) for a, b in zip(got, again))
            more = max(more, launches)
            # an output that is not asked for keeps what it holds, and the others are as they were
            some = s.run(qat, True, (False, True, False))
            assert bool((some[0] == -7.0).all()) and bool((some[2] == -7.0).all())
            assert float((some[1].double() - got[1].double()).norm()) <= 1e-4 * float(got[1].double().norm())
            if qat:
                some = s.run(qat, True, (True, False, False))
                s.check([some[0]], qat)
                assert bool((some[1] == -7.0).all()) and bool((some[2] == -7.0).all())
        assert lords.lords_poll_status() == 0
    assert more > 3          # parts were taken: one part is three launches, four where rows are copied
    workspace(64 * n * 2 - 256)
    out = [torch.full(t, -7.0, device="cuda") for t in ((m, r), (r, n))]
    with pytest.raises(lords.LordsError) as e:
        lords.lords_linear_backward_factors_checkpoint(s.g, s.cq, s.ce, s.q, s.B, s.A, s.cb, bits, M, m, n, r, *out)
    torch.cuda.synchronize()
    assert e.value.status == -9 and all(bool((t == -7.0).all()) for t in out)


def test_gradients_in_parts_are_captured(workspace):
    s = Step(256, 512, 8, 300, 4, 3)
    workspace(300 << 10)
    want = s.run(True, True)
    torch.cuda.synchronize()
    M, m, n, r = s.sizes
    dW, dB, dA = torch.empty(m, n, device="cuda"), torch.empty(m, r, device="cuda"), torch.empty(r, n, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lords.lords_linear_backward_qat_checkpoint(s.g, s.cq, s.ce, s.W, s.q, s.B, s.A, s.cb, s.bits, M, m, n, r, dW, dB, dA)
    for _ in range(3):
        for t in (dW, dB, dA):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dW, dB, dA), want))


@pytest.mark.parametrize("M", [8192, 10000])
def test_long_sequences_keep_their_schedule(M):
    """The default workspace: 8192 tokens of 14336 columns leave no room for the contributions, 10000 do not fit at all."""
    s = Step(4096, 14336, 32, M, 4, 1)
    got = s.run(False, True)
    assert lords.lords_last_path() == "backward_tensor"
    s.check(got, False)
    del got
    got = s.run(True, True)
    assert lords.lords_last_path() == "backward_qat_tensor"
    s.check(got, True)
