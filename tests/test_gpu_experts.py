"""Products and factors of a layer of experts against their formulas in float64.

Bounds, element by element.  A sum of K products in fp32 in any order, with additions that may be truncated, is off by at most
(K + 2) 2^-23 S, S the sum of the products' magnitudes (products of bf16 values are exact); one rounding to bf16 adds 2^-8 of the result.  A running
average adds three fp32 roundings of its terms.
"""
import numpy as np
import pytest
import torch

from paper_2007_00784_amd import kfac as K
from gpu_util import Ctx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(64 << 20)
    yield c
    c.close()


def near(got, want, mags, terms, bf16):
    """got (device) against want, with mags the sums of magnitudes (float64, CPU)."""
    got = got.double().cpu()
    bound = (terms + 2) * 2.0 ** -23 * mags + (2.0 ** -8 if bf16 else 2.0 ** -23) * want.abs() + 1e-37
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got - want).abs() / bound).max()))


class Layer:
    """Samples and weights of one layer; every matrix of samples lies in a larger buffer with a pitch and a start of its own."""

    def __init__(self, counts, d_in, d_out, ones=0, bf16=True, lead=0, behind=0, pad=0, start=0, seed=0, dev="cuda:0"):
        self.gen = torch.Generator().manual_seed(seed + 7919 * d_in + 31 * d_out + len(counts))
        self.dt = torch.bfloat16 if bf16 else torch.float32
        self.bf16, self.dev, self.pad, self.start = bf16, dev, pad, start
        self.E, self.d_in, self.d_out, self.ones = len(counts), d_in, d_out, ones
        off = [lead]
        for c in counts:
            off.append(off[-1] + c)
        self.off, self.R = off, off[-1] + behind
        self.offsets = torch.tensor(off, dtype=torch.int32, device=dev)
        self.W = torch.randn((self.E, d_out, d_in + ones), generator=self.gen).to(self.dt)
        self.Wd = self.W.to(dev)

    def samples(self, d, fill=None, garbage=float("nan")):
        """(device view, float64 copy): rows that belong to nobody hold garbage."""
        pitch = d + self.pad
        buf = torch.full((self.start + self.R * pitch,), 0.0)
        view = torch.as_strided(buf, (self.R, d), (pitch, 1), self.start)
        view.copy_(torch.randn((self.R, d), generator=self.gen) if fill is None else torch.full((self.R, d), fill))
        if fill is None:
            view[:self.off[0]] = garbage
            view[self.off[-1]:] = garbage
        gap = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(gap, (self.R, d), (pitch, 1), self.start).fill_(False)
        buf[gap] = garbage if fill is None else fill
        b = buf.to(self.dt).to(self.dev)
        host = b.cpu().double()
        return torch.as_strided(b, (self.R, d), (pitch, 1), self.start), torch.as_strided(host, (self.R, d), (pitch, 1), self.start), b

    def parts(self):
        return [(e, self.off[e], self.off[e + 1]) for e in range(self.E) if self.off[e + 1] > self.off[e]]


# counts, d_in, d_out, ones: every side at 1, below, at and above the eight of a group, the 64 of a slab and the 128 and 256 of a tile
SHAPES = [
    ([3], 8, 8, 0),
    ([1], 64, 16, 1),
    ([0, 1, 0, 2, 0], 72, 40, 0),
    ([5, 0, 7], 1, 9, 1),
    ([4, 3], 9, 1, 0),
    ([2, 9], 7, 5, 1),
    ([17, 1, 64], 65, 71, 1),
    ([70, 0, 5], 128, 257, 0),
    ([130, 61], 199, 255, 1),
    ([257, 3], 264, 264, 1),
    ([300, 0, 513], 130, 513, 0),
    ([1] * 70 + [0] * 70 + [3] * 5, 16, 24, 1),     # more experts than a wave has lanes
]
STYLES = [dict(), dict(lead=3, behind=5, pad=8), dict(behind=2, pad=3, start=1)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("style", range(len(STYLES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_products(ctx, shape, style, bf16):
    counts, d_in, d_out, ones = SHAPES[shape]
    L = Layer(counts, d_in, d_out, ones, bf16, **STYLES[style])
    X, Xh, _ = L.samples(d_in)
    G, Gh, _ = L.samples(d_out)
    Y, _, Yb = L.samples(d_out, fill=7.0)
    dX, _, dXb = L.samples(d_in, fill=7.0)
    dW = torch.full((L.E, d_out, d_in + ones), float("nan"), device=L.dev)
    K.kfac_experts_forward(ctx.h, X, L.Wd, L.offsets, Y, append_ones=ones)
    K.kfac_experts_input_grad(ctx.h, G, L.Wd, L.offsets, dX, append_ones=ones)
    K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=ones)
    torch.cuda.synchronize()
    W = L.W.double()
    want, mags = torch.zeros(L.E, d_out, d_in + ones, dtype=torch.float64), torch.zeros(L.E, d_out, d_in + ones, dtype=torch.float64)
    for e, a, b in L.parts():
        w = W[e, :, :d_in]
        bias = W[e, :, d_in] if ones else torch.zeros(d_out, dtype=torch.float64)
        near(Y[a:b], Xh[a:b] @ w.T + bias, Xh[a:b].abs() @ w.abs().T + bias.abs(), d_in + 1, bf16)
        near(dX[a:b], Gh[a:b] @ w, Gh[a:b].abs() @ w.abs(), d_out, bf16)
        x = torch.cat([Xh[a:b], torch.ones(b - a, 1, dtype=torch.float64)], 1) if ones else Xh[a:b]
        want[e], mags[e] = Gh[a:b].T @ x, Gh[a:b].abs().T @ x.abs()
    near(dW, want, mags, max(counts), False)
    for t, buf in ((Y, Yb), (dX, dXb)):                 # what belongs to nobody is as it was
        t[L.off[0]:L.off[-1]] = 7.0
        assert bool((buf == 7.0).all())


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_weight_grad_in_bf16_and_accumulated(ctx, shape, bf16):
    counts, d_in, d_out, ones = SHAPES[shape]
    L = Layer(counts, d_in, d_out, ones, bf16)
    X, Xh, _ = L.samples(d_in)
    G, Gh, _ = L.samples(d_out)
    n = torch.zeros(L.E, d_out, d_in + ones, dtype=torch.float64)
    want, mags = n.clone(), n.clone()
    for e, a, b in L.parts():
        x = torch.cat([Xh[a:b], torch.ones(b - a, 1, dtype=torch.float64)], 1) if ones else Xh[a:b]
        want[e], mags[e] = Gh[a:b].T @ x, Gh[a:b].abs().T @ x.abs()
    for dt in (torch.float32, torch.bfloat16):
        first = torch.randn(n.shape, generator=L.gen).to(dt)
        for acc in (False, True):
            dW = first.to(L.dev).clone()
            K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=ones, accumulate=acc)
            w = want + (first.double() if acc else 0.0)
            near(dW, w, mags + (first.double().abs() if acc else 0.0), max(counts) + 1, dt is torch.bfloat16)


FACTOR_SHAPES = [([3], 8, 0), ([0, 5, 0, 1], 16, 1), ([40, 7], 5, 1), ([2, 3], 1, 0), ([70, 130], 72, 1), ([200, 0, 64], 133, 1), ([65, 300], 257, 0),
                 ([90, 33], 300, 1), ([1] * 66, 24, 1)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("style", range(len(STYLES)))
@pytest.mark.parametrize("shape", range(len(FACTOR_SHAPES)))
def test_factors(ctx, shape, style, bf16):
    counts, d, ones = FACTOR_SHAPES[shape]
    L = Layer(counts, d, 1, ones, bf16, **STYLES[style])
    X, Xh, _ = L.samples(d)
    D = d + ones
    h = torch.randn((L.E, D, D), generator=L.gen)
    F0 = h + h.transpose(1, 2)
    for mean, scale, decay in ((True, 1.0, 0.95), (False, 0.3, 0.0), (True, 2.0, 0.0), (False, 0.7, 0.5), (True, 1.0, 1.0)):
        F = F0.to(L.dev).clone()
        if decay == 0.0 and not mean:
            F.fill_(float("nan"))                       # decay 0 overwrites whatever was there
        K.kfac_update_factors_experts(ctx.h, X, L.offsets, F, append_ones=ones, scale=scale, decay=decay, mean=mean)
        again = F0.to(L.dev).clone()
        K.kfac_update_factors_experts(ctx.h, X, L.offsets, again, append_ones=ones, scale=scale, decay=decay, mean=mean)
        torch.cuda.synchronize()
        assert torch.equal(F, F.transpose(1, 2)) and torch.equal(F, again)
        want, mags = torch.zeros(L.E, D, D, dtype=torch.float64), torch.zeros(L.E, D, D, dtype=torch.float64)
        for e in range(L.E):
            a, b = L.off[e], L.off[e + 1]
            if a == b and mean:
                want[e] = F0[e].double()
                continue
            x = torch.cat([Xh[a:b], torch.ones(b - a, 1, dtype=torch.float64)], 1) if ones else Xh[a:b]
            c = (1.0 - decay) * scale / (b - a if mean else 1)
            want[e] = decay * F0[e].double() + c * (x.T @ x)
            mags[e] = decay * F0[e].double().abs() + c * (x.abs().T @ x.abs())
        near(F, want, mags, max(counts) + 4, False)


def test_offsets_are_clamped(ctx):
    """Offsets outside the samples, and descending ones, touch nothing outside; rows that only valid offsets name come out right."""
    L = Layer([4, 4, 4], 72, 40, behind=4)
    X, Xh, _ = L.samples(72, garbage=1.0)
    for off in ([-5, 4, 8, 1000], [0, 4, 4, 2 ** 31 - 1], [-2 ** 31, -7, 4, 12], [0, 16, 3, 12], [16, 16, 16, 16]):
        o = torch.tensor(off, dtype=torch.int32, device=L.dev)
        Y, _, buf = L.samples(40, fill=7.0)
        dW = torch.full((3, 40, 72), float("nan"), device=L.dev)
        F = torch.zeros((3, 72, 72), device=L.dev)
        K.kfac_experts_forward(ctx.h, X, L.Wd, o, Y)
        K.kfac_experts_weight_grad(ctx.h, Y, X, o, dW)
        K.kfac_update_factors_experts(ctx.h, X, o, F, mean=False)
        torch.cuda.synchronize()
        clamped = [min(max(v, 0), L.R) for v in off]
        if all(a <= b for a, b in zip(clamped, clamped[1:])):
            for e in range(3):
                a, b = clamped[e], clamped[e + 1]
                w = L.W[e].double()
                if b > a:
                    near(Y[a:b], Xh[a:b] @ w.T, Xh[a:b].abs() @ w.abs().T, 72, True)
                near(F[e], Xh[a:b].T @ Xh[a:b], Xh[a:b].abs().T @ Xh[a:b].abs(), 16, False)
        assert bool(torch.isfinite(dW).all())


def test_what_is_not_finite_stays_with_its_row(ctx):
    """Inf and NaN in one row, or in one expert's weights, reach that row's or that expert's results only."""
    L = Layer([70, 90, 33], 200, 136, ones=1)
    X, Xh, _ = L.samples(200)
    X[75, 3], X[76, 199] = float("inf"), float("nan")
    L.Wd[2, 5, 7] = float("inf")
    Y, _, _ = L.samples(136, fill=0.0)
    dX, _, _ = L.samples(200, fill=0.0)
    K.kfac_experts_forward(ctx.h, X, L.Wd, L.offsets, Y, append_ones=True)
    G, _, _ = L.samples(136)
    K.kfac_experts_input_grad(ctx.h, G, L.Wd, L.offsets, dX, append_ones=True)
    dW = torch.zeros((3, 136, 201), device=L.dev)
    K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=True)
    rows = torch.isfinite(Y).all(1)
    assert not rows[75] and not rows[76] and bool(rows[:75].all()) and bool(rows[77:160].all())
    assert bool((~torch.isfinite(Y[160:])).any(1).all()) and bool(torch.isfinite(Y[160:, :5]).all()) and bool(torch.isfinite(Y[160:, 6:]).all())
    assert bool(torch.isfinite(dX[:160]).all()) and bool(torch.isfinite(dX[160:, :7]).all()) and bool(torch.isfinite(dX[160:, 8:]).all())
    assert bool(torch.isfinite(dW[0]).all()) and bool(torch.isfinite(dW[2]).all())
    assert bool(torch.isfinite(dW[1][:, :3]).all()) and bool(torch.isfinite(dW[1][:, 200]).all())


def test_weight_gradient_against_differences(ctx):
    """sum(C * Y) as a function of W and X: the gradients by the two calls against central differences of the formula in float64."""
    L = Layer([9, 0, 14], 24, 16, ones=1, bf16=False)
    X, Xh, _ = L.samples(24)
    C, Ch, _ = L.samples(16)
    dW = torch.zeros((3, 16, 25), device=L.dev)
    dX, _, _ = L.samples(24, fill=0.0)
    K.kfac_experts_weight_grad(ctx.h, C, X, L.offsets, dW, append_ones=True)
    K.kfac_experts_input_grad(ctx.h, C, L.Wd, L.offsets, dX, append_ones=True)

    def loss(W, x):
        return sum(float((Ch[a:b] * (torch.cat([x[a:b], torch.ones(b - a, 1, dtype=torch.float64)], 1) @ W[e].T)).sum()) for e, a, b in L.parts())

    W = L.W.double()
    for seed in range(4):                                # the loss is linear in either: a difference along a direction is exact
        g = torch.Generator().manual_seed(seed)
        V, U = torch.randn(W.shape, generator=g, dtype=torch.float64), torch.randn(Xh.shape, generator=g, dtype=torch.float64)
        dv, du = (loss(W + V, Xh) - loss(W - V, Xh)) / 2, (loss(W, Xh + U) - loss(W, Xh - U)) / 2
        # each gradient is off by 32 * 2^-23 of its magnitudes at most, summed over 3 * 16 * 25 and 23 * 24 entries of size one
        assert abs(float((dW.cpu().double() * V).sum()) - dv) <= 32 * 2.0 ** -23 * 1200 * 40
        assert abs(float((dX.cpu().double() * U).sum()) - du) <= 32 * 2.0 ** -23 * 552 * 40


@pytest.mark.parametrize("bf16", [True, False])
def test_captured_calls_read_the_offsets_of_each_replay(bf16):
    s = torch.cuda.Stream()
    dev = torch.device("cuda:0")
    L = Layer([40, 0, 90], 72, 136, ones=1, bf16=bf16)
    X, Xh, _ = L.samples(72)
    G, Gh, _ = L.samples(136)
    Y, _, _ = L.samples(136, fill=0.0)
    dX, _, _ = L.samples(72, fill=0.0)
    dW = torch.zeros((3, 136, 73), device=dev)
    F = torch.zeros((3, 73, 73), device=dev)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    h = K.kfac_create(0, s.cuda_stream, ws)
    torch.cuda.synchronize()

    def calls():
        K.kfac_experts_forward(h, X, L.Wd, L.offsets, Y, append_ones=True)
        K.kfac_experts_input_grad(h, G, L.Wd, L.offsets, dX, append_ones=True)
        K.kfac_experts_weight_grad(h, G, X, L.offsets, dW, append_ones=True)
        K.kfac_update_factors_experts(h, X, L.offsets, F, append_ones=True, decay=0.0)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls()
    for off in ([0, 40, 40, 130], [0, 1, 100, 130], [0, 0, 0, 130], [10, 30, 31, 32]):
        L.offsets.copy_(torch.tensor(off, dtype=torch.int32))
        for t in (Y, dX, dW, F):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dX, dW, F)]
        for t in (Y, dX, dW, F):
            t.zero_()
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        for a, b in zip(got, (Y, dX, dW, F)):
            assert torch.equal(a, b)
        L.off = off
        for e, a, b in L.parts():
            near(got[0][a:b], Xh[a:b] @ L.W[e, :, :72].double().T + L.W[e, :, 72].double(),
                 Xh[a:b].abs() @ L.W[e, :, :72].double().abs().T + L.W[e, :, 72].double().abs(), 73, bf16)
    K.kfac_destroy(h)


def test_no_rows(ctx):
    off = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    X = torch.empty((0, 16), dtype=torch.bfloat16, device="cuda:0")
    G = torch.empty((0, 24), dtype=torch.bfloat16, device="cuda:0")
    W = torch.ones((2, 24, 16), dtype=torch.bfloat16, device="cuda:0")
    K.kfac_experts_forward(ctx.h, X, W, off, G)
    K.kfac_experts_input_grad(ctx.h, G, W, off, X)
    dW = torch.ones((2, 24, 16), device="cuda:0")
    K.kfac_experts_weight_grad(ctx.h, G, X, off, dW, accumulate=True)
    assert bool((dW == 1).all())
    K.kfac_experts_weight_grad(ctx.h, G, X, off, dW)
    assert bool((dW == 0).all())
    F = torch.ones((2, 16, 16), device="cuda:0")
    K.kfac_update_factors_experts(ctx.h, X, off, F, decay=0.5)
    assert bool((F == 1).all())
    K.kfac_update_factors_experts(ctx.h, X, off, F, decay=0.5, mean=False)
    assert bool((F == 0.5).all())


# ---- every engine that a call can take, whole and in parts ----
FORWARD, INPUT_GRAD, WEIGHT_GRAD, FACTORS = range(4)
FEW, SOME, SMALL, WIDE, WIDE_SMALL, TILES, MEDIUM = range(7)
# mode, counts, d_in, d_out, ones, bf16, engine, parts
ENGINES = [
    (FORWARD, [3, 0, 5], 265, 130, 1, True, FEW, False),
    (FORWARD, [300, 200], 75, 523, 1, True, SOME, False),
    (FORWARD, [9000, 1, 2999], 18, 1101, 1, True, WIDE, False),
    (FORWARD, [100] * 39 + [77], 301, 1100, 0, True, WIDE_SMALL, False),
    (INPUT_GRAD, [150] * 20 + [0] + [163] * 19, 1001, 27, 0, True, WIDE, False),
    (INPUT_GRAD, [200, 3, 97], 301, 130, 1, True, WIDE_SMALL, False),
    (INPUT_GRAD, [170, 130], 70, 1607, 1, True, WIDE_SMALL, True),
    (WEIGHT_GRAD, [100] * 20 + [0] + [101] * 19, 1003, 133, 1, True, WIDE, False),
    (WEIGHT_GRAD, [50, 40], 300, 140, 1, True, WIDE_SMALL, False),
    (WEIGHT_GRAD, [4100, 0, 60, 130], 75, 131, 1, True, WIDE_SMALL, True),
    (FACTORS, [1500] * 8, 1601, 1, 1, True, WIDE, False),
    (FACTORS, [50, 40], 300, 1, 1, True, WIDE_SMALL, False),
    (FACTORS, [6100, 160], 203, 1, 1, True, WIDE_SMALL, True),
    (FORWARD, [40, 21], 75, 133, 1, False, SMALL, False),
    (FORWARD, [12000], 16, 130, 1, False, TILES, False),
    (FORWARD, [2205], 1001, 1103, 1, False, MEDIUM, False),
    (FORWARD, [30, 0, 7], 70, 1103, 1, False, SMALL, False),
    (FORWARD, [3] * 12 + [1], 70, 1607, 1, False, MEDIUM, False),
    (FORWARD, [200, 103], 300, 3, 1, False, TILES, True),
    (FORWARD, [8000], 1601, 603, 1, False, TILES, True),
    (INPUT_GRAD, [40, 21], 75, 133, 1, False, SMALL, False),
    (INPUT_GRAD, [2200], 1603, 29, 1, False, TILES, False),
    (INPUT_GRAD, [2205], 1103, 1001, 1, False, MEDIUM, False),
    (INPUT_GRAD, [3] * 12 + [1], 1001, 75, 1, False, MEDIUM, False),
    (INPUT_GRAD, [300], 3, 1607, 1, False, TILES, True),
    (WEIGHT_GRAD, [40, 21], 75, 133, 1, False, SMALL, False),
    (WEIGHT_GRAD, [4] * 40, 1601, 101, 1, False, TILES, False),
    (WEIGHT_GRAD, [190, 0, 103] * 8, 1601, 75, 1, False, MEDIUM, False),
    (WEIGHT_GRAD, [6600], 75, 133, 1, False, TILES, True),
    (FACTORS, [40, 21], 135, 1, 1, False, SMALL, False),
    (FACTORS, [4, 3, 5], 603, 1, 1, False, SMALL, False),
    (FACTORS, [4, 9, 3, 5, 0, 6, 5, 5], 513, 1, 1, False, TILES, False),
    (FACTORS, [9900, 700], 255, 1, 1, False, TILES, True),
]


def plan_of(mode, L, workspace):
    import ctypes
    f = K.lib().kfac_experts_plan
    f.argtypes = [ctypes.c_int, ctypes.POINTER(K.kfac_expert_desc), ctypes.c_size_t]
    d = K.kfac_expert_desc(L.E, L.R, L.d_in, L.d_out, L.ones, K.KFAC_BF16 if L.bf16 else K.KFAC_F32, 4096)
    p = f(mode, ctypes.byref(d), workspace)
    return p // 100, p % 100


def near_gpu(got, want, mags, terms, bf16):
    bound = (terms + 2) * 2.0 ** -23 * mags + (2.0 ** -8 if bf16 else 2.0 ** -23) * want.abs() + 1e-37
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("case", range(len(ENGINES)))
def test_engines(ctx, case):
    mode, counts, d_in, d_out, ones, bf16, engine, parts = ENGINES[case]
    L = Layer(counts, d_in, d_out, ones, bf16, behind=3, seed=case)
    room = K.kfac_experts_workspace_bytes(L.E, L.R, d_in, d_out, ones, K.KFAC_BF16 if bf16 else K.KFAC_F32)
    assert room <= ctx.ws.numel()
    got_engine, got_parts = plan_of(mode, L, room)
    assert (got_engine, got_parts > 1) == (engine, parts) and plan_of(mode, L, ctx.ws.numel()) == (got_engine, got_parts)
    bare = K.kfac_create(0, ctx.stream.cuda_stream, None)
    for h in (ctx.h, bare):
        X, Xh, _ = L.samples(d_in)
        G, Gh, _ = L.samples(d_out)
        Xd, Gd, W = X.double(), G.double(), L.Wd.double()
        if mode in (FORWARD, INPUT_GRAD):
            out, _, buf = L.samples(d_out if mode == FORWARD else d_in, fill=7.0)
            if mode == FORWARD:
                K.kfac_experts_forward(h, X, L.Wd, L.offsets, out, append_ones=ones)
            else:
                K.kfac_experts_input_grad(h, G, L.Wd, L.offsets, out, append_ones=ones)
            for e, a, b in L.parts():
                w = W[e, :, :d_in].contiguous()
                if mode == FORWARD:
                    bias = W[e, :, d_in] if ones else torch.zeros(d_out, dtype=torch.float64, device=L.dev)
                    wt = w.t().contiguous()
                    near_gpu(out[a:b], Xd[a:b] @ wt + bias, Xd[a:b].abs() @ wt.abs() + bias.abs(), d_in + 1, bf16)
                else:
                    near_gpu(out[a:b], Gd[a:b] @ w, Gd[a:b].abs() @ w.abs(), d_out, bf16)
            out[:L.off[-1]] = 7.0
            assert bool((buf == 7.0).all())
        else:
            rows = G if mode == WEIGHT_GRAD else X
            D = d_in + ones
            out = torch.full((L.E, d_out if mode == WEIGHT_GRAD else D, D), 1.0, device=L.dev)
            if mode == WEIGHT_GRAD:
                K.kfac_experts_weight_grad(h, G, X, L.offsets, out, append_ones=ones, accumulate=True)
            else:
                K.kfac_update_factors_experts(h, X, L.offsets, out, append_ones=ones, scale=0.5, decay=0.25)
            for e in range(L.E):
                a, b = L.off[e], L.off[e + 1]
                x = torch.cat([Xd[a:b], torch.ones(b - a, 1, dtype=torch.float64, device=L.dev)], 1) if ones else Xd[a:b]
                r = (Gd[a:b] if mode == WEIGHT_GRAD else x).t().contiguous()
                if mode == WEIGHT_GRAD:
                    near_gpu(out[e], 1.0 + r @ x, 1.0 + r.abs() @ x.abs(), b - a + 2, False)
                elif b > a:
                    c = 0.75 * 0.5 / (b - a)
                    near_gpu(out[e], 0.25 + c * (r @ x), 0.25 + c * (r.abs() @ x.abs()), b - a + 4, False)
                    assert torch.equal(out[e], out[e].t())
                else:
                    assert bool((out[e] == 1).all())
    torch.cuda.synchronize()
    K.kfac_destroy(bare)


def test_descending_offsets_with_parts(ctx):
    """Descending offsets name more rows than there are, and more tiles than the workspace was sized for: nothing outside is touched, and the next
    call is as it should be."""
    L = Layer([170, 130], 70, 1607, 1, True)
    assert plan_of(INPUT_GRAD, L, ctx.ws.numel())[1] > 1
    G, Gh, _ = L.samples(1607)
    dX, _, buf = L.samples(70, fill=7.0)
    room = K.kfac_experts_workspace_bytes(2, 300, 70, 1607, 1, K.KFAC_BF16)
    ws = torch.full((room + (32 << 20),), 0x5a, dtype=torch.uint8, device=L.dev)
    h = K.kfac_create(0, ctx.stream.cuda_stream, ws, room)
    for off in ([0, 300, 0], [300, 0, 300], [0, 2 ** 31 - 1, -5]):
        K.kfac_experts_input_grad(h, G, L.Wd, torch.tensor(off, dtype=torch.int32, device=L.dev), dX, append_ones=True)
    torch.cuda.synchronize()
    assert bool((ws[room:] == 0x5a).all())
    K.kfac_experts_input_grad(h, G, L.Wd, L.offsets, dX, append_ones=True)
    for e, a, b in L.parts():
        w = L.W[e, :, :70].double()
        near(dX[a:b], Gh[a:b] @ w, Gh[a:b].abs() @ w.abs(), 1607, True)
    torch.cuda.synchronize()
    K.kfac_destroy(h)


def test_a_short_side_over_many_rows(ctx):
    """bf16 with a side below the sixteen bytes of a group, over so many rows that the sum goes in parts."""
    for d_in, d_out in ((5, 40), (40, 3)):
        L = Layer([9000], d_in, d_out, 1, True)
        assert plan_of(WEIGHT_GRAD, L, ctx.ws.numel()) [0] == TILES and plan_of(WEIGHT_GRAD, L, ctx.ws.numel())[1] > 1
        X, Xh, _ = L.samples(d_in)
        G, Gh, _ = L.samples(d_out)
        dW = torch.zeros((1, d_out, d_in + 1), device=L.dev)
        K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=True)
        x = torch.cat([Xh, torch.ones(9000, 1, dtype=torch.float64)], 1)
        near(dW[0], Gh.T @ x, Gh.abs().T @ x.abs(), 9000, False)


def test_another_stream_than_the_callers(ctx):
    """A context on a stream of its own, with work on it before and behind the calls; two contexts side by side."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    L = Layer([300, 0, 200], 130, 264, 1, True)
    X, Xh, _ = L.samples(130)
    hs = [K.kfac_create(0, s.cuda_stream, torch.empty(8 << 20, dtype=torch.uint8, device=L.dev)) for s in streams]
    outs = []
    torch.cuda.synchronize()
    for s, h in zip(streams, hs):
        with torch.cuda.stream(s):
            x = torch.zeros_like(X)
            big = torch.randn(2000, 2000, device=L.dev)
            for _ in range(4):
                big = big @ big / 2000
            x.copy_(X)
            y = torch.zeros((L.R, 264), dtype=L.dt, device=L.dev)
            K.kfac_experts_forward(h, x, L.Wd, L.offsets, y, append_ones=True)
            outs.append(y.clone())
    torch.cuda.synchronize()
    for e, a, b in L.parts():
        w = L.W[e].double()
        near(outs[0][a:b], Xh[a:b] @ w[:, :130].T + w[:, 130], Xh[a:b].abs() @ w[:, :130].abs().T + w[:, 130].abs(), 131, True)
    assert torch.equal(outs[0], outs[1])
    for h in hs:
        K.kfac_destroy(h)


def test_more_experts_than_a_wave(ctx):
    """300 experts, most of them without rows: prefix sums over several waves' worth of offsets."""
    counts = [(i * 7919) % 11 if i % 3 == 0 else 0 for i in range(300)]
    for bf16 in (True, False):
        L = Layer(counts, 40, 24, 1, bf16)
        X, Xh, _ = L.samples(40)
        G, Gh, _ = L.samples(24)
        Y, _, _ = L.samples(24, fill=0.0)
        dW = torch.full((300, 24, 41), float("nan"), device=L.dev)
        F = torch.ones((300, 41, 41), device=L.dev)
        K.kfac_experts_forward(ctx.h, X, L.Wd, L.offsets, Y, append_ones=True)
        K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=True)
        K.kfac_update_factors_experts(ctx.h, X, L.offsets, F, append_ones=True)
        for e in range(300):
            a, b = L.off[e], L.off[e + 1]
            if a == b:
                assert bool((dW[e] == 0).all()) and bool((F[e] == 1).all())
                continue
            x = torch.cat([Xh[a:b], torch.ones(b - a, 1, dtype=torch.float64)], 1)
            w = L.W[e].double()
            near(Y[a:b], x @ w.T, x.abs() @ w.abs().T, 41, bf16)
            near(dW[e], Gh[a:b].T @ x, Gh[a:b].abs().T @ x.abs(), b - a, False)
            near(F[e], x.T @ x / (b - a), x.abs().T @ x.abs() / (b - a), b - a + 4, False)
