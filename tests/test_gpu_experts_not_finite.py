"""Infinities and NaN in products and factors of a layer of experts, through every kernel that a call can take, whole and in parts: they reach the
sums that they belong to, and every other element is bit for bit what it is without them.  (Padding is multiplied with zeros that were
loaded as such, never with what lies there.)"""
import pytest
import torch

from paper_2007_00784_amd import kfac as K
from gpu_util import Ctx
from test_gpu_experts import ENGINES, FACTORS, FORWARD, INPUT_GRAD, WEIGHT_GRAD, Layer, plan_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(64 << 20)
    yield c
    c.close()


@pytest.mark.parametrize("case", range(len(ENGINES)))
def test_every_engine(ctx, case):
    mode, counts, d_in, d_out, ones, bf16, engine, parts = ENGINES[case]
    L = Layer(counts, d_in, d_out, ones, bf16, behind=3, seed=case)      # (the rows behind the last expert are NaN from the start)
    assert plan_of(mode, L, ctx.ws.numel())[0] == engine and (plan_of(mode, L, ctx.ws.numel())[1] > 1) == parts
    X, _, _ = L.samples(d_in)
    G, _, _ = L.samples(d_out)
    (e0, _, end), (e1, beg, _) = L.parts()[0], L.parts()[-1]              # the last row of the first expert, the first row of the last
    D = d_in + ones
    bare = K.kfac_create(0, ctx.stream.cuda_stream, None)

    def call(h):
        if mode in (FORWARD, INPUT_GRAD):
            out = torch.zeros((L.R, d_out if mode == FORWARD else d_in), dtype=L.dt, device=L.dev)
            if mode == FORWARD:
                K.kfac_experts_forward(h, X, L.Wd, L.offsets, out, append_ones=ones)
            else:
                K.kfac_experts_input_grad(h, G, L.Wd, L.offsets, out, append_ones=ones)
        else:
            out = torch.ones((L.E, d_out if mode == WEIGHT_GRAD else D, D), device=L.dev)
            if mode == WEIGHT_GRAD:
                K.kfac_experts_weight_grad(h, G, X, L.offsets, out, append_ones=ones, accumulate=True)
            else:
                K.kfac_update_factors_experts(h, X, L.offsets, out, append_ones=ones, decay=0.25)
        return out

    clean = [call(h) for h in (ctx.h, bare)]
    hit = torch.zeros_like(clean[0], dtype=torch.bool)
    nan, inf = float("nan"), float("inf")
    if mode in (FORWARD, INPUT_GRAD):
        a = X if mode == FORWARD else G
        a[end - 1, -1], a[beg, 0] = nan, inf                              # (the last column lies in a group that is shifted where K is no multiple of it)
        L.Wd[e1, d_out - 1, d_in - 1] = -inf
        hit[[end - 1, beg]] = True
        hit[beg:L.off[-1], -1] = True
    elif mode == WEIGHT_GRAD:
        X[end - 1, -1], G[beg, 0] = nan, inf
        hit[e0, :, d_in - 1] = True
        hit[e1, 0] = True
    else:
        X[end - 1, -1], X[beg, 0] = nan, inf
        for e, c in ((e0, d_in - 1), (e1, 0)):
            hit[e, c] = True
            hit[e, :, c] = True
    for h, was in zip((ctx.h, bare), clean):
        got = call(h)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(was).all())
        assert not bool(torch.isfinite(got[hit]).any())
        assert torch.equal(got[~hit], was[~hit])
    K.kfac_destroy(bare)


@pytest.mark.parametrize("bf16", [True, False])
def test_the_neighbour_behind_the_last_row(ctx, bf16):
    """Experts of 1 to 40 rows whose neighbours are NaN throughout: sums over rows end inside a slab, and what follows belongs to the next expert."""
    counts = [r for n in range(1, 41) for r in (n, 3)]
    L = Layer(counts, 24, 16, 1, bf16)
    X, _, _ = L.samples(24)
    G, _, _ = L.samples(16)

    def call():
        dW, F = torch.zeros((L.E, 16, 25), device=L.dev), torch.zeros((L.E, 25, 25), device=L.dev)
        Y, dX = torch.zeros((L.R, 16), dtype=L.dt, device=L.dev), torch.zeros((L.R, 24), dtype=L.dt, device=L.dev)
        K.kfac_experts_forward(ctx.h, X, L.Wd, L.offsets, Y, append_ones=True)
        K.kfac_experts_input_grad(ctx.h, G, L.Wd, L.offsets, dX, append_ones=True)
        K.kfac_experts_weight_grad(ctx.h, G, X, L.offsets, dW, append_ones=True)
        K.kfac_update_factors_experts(ctx.h, X, L.offsets, F, append_ones=True)
        return dW, F, Y, dX

    clean = call()
    own = torch.zeros(L.R, dtype=torch.bool)
    for e, a, b in L.parts():
        own[a:b] = e % 2 == 0
    X[~own], G[~own] = float("nan"), float("nan")
    got = call()
    torch.cuda.synchronize()
    for a, b in zip(got[:2], clean[:2]):
        assert torch.equal(a[::2], b[::2])
    for a, b in zip(got[2:], clean[2:]):
        assert torch.equal(a[own], b[own])
