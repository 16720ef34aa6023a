"""Tokens to experts and back where a training batch is: more experts' rows than the caches hold, copies behind a sort of many slots at every number of lanes,
batches of more workgroups than one launch has, and ids that name an expert more than once.  All against float64 (on the GPU: the sizes are large).

Bounds as in test_gpu_tokens.py: a sum of K terms by fma is off by (K + 2) 2^-24 of their magnitudes' sum, a rounding to the output's type by half a step.
"""
import math

import pytest
import torch

from paper_2007_00784_amd import kfac as K
from gpu_util import Ctx
from test_gpu_tokens import DEV, STYLES, U, choice, half_step, logits_for, matrix, near, order_of, random_ids, softmax, spread, weights_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(8 << 20)
    yield c
    c.close()
    torch.cuda.empty_cache()


def padded(R, d, dt, pad=0, start=0, fill=5.0):
    """(a view [R, d] of a buffer with a pitch and a start of its own, the buffer, which of its elements are not the view's)"""
    buf = torch.full((start + R * (d + pad),), fill, dtype=dt, device=DEV)
    other = torch.ones(buf.shape, dtype=torch.bool, device=DEV)
    torch.as_strided(other, (R, d), (d + pad, 1), start).fill_(False)
    return torch.as_strided(buf, (R, d), (d + pad, 1), start), buf, other


def close(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound + 1e-37)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


# T, k, E, d: over 128 MB of experts' rows in bf16; 8 to 256 lanes a token, 1024 for few tokens, one, two and four rows at a time and what is left of four
LARGE = [(70000, 1, 8, 1031), (18000, 2, 8, 2051), (9000, 4, 40, 2050), (6100, 6, 64, 2049), (4000, 7, 5, 5003), (250, 8, 16, 33003), (60000, 3, 64, 601), (90000, 5, 20, 203), (300000, 4, 16, 73),
         (50000, 3, 9, 500)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("shape", range(len(LARGE)))
def test_more_rows_than_the_caches_hold(ctx, shape, bf16):
    T, k, E, d = LARGE[shape]
    dt, style = torch.bfloat16 if bf16 else torch.float32, STYLES[shape % 3]
    assert T * k * d * (2 if bf16 else 4) > 128e6
    gen, dgen = torch.Generator().manual_seed(shape), torch.Generator(device=DEV).manual_seed(shape)
    new = lambda *s: torch.randn(*s, generator=dgen, device=DEV)  # noqa: E731
    ids = random_ids(T, k, E, gen)
    rows, used = order_of(ids, E)[1].to(DEV), int(order_of(ids, E)[0][-1])
    has, R = rows >= 0, T * k + shape % 4
    at = rows.clamp(min=0).long()
    Ys = padded(R, d, dt, fill=math.nan, **style)[0]
    Ys[:used] = new(used, d).to(dt)
    a, g, w = new(T, d).to(dt), new(T, d).to(dt), new(T, k)
    w[~has] = math.nan
    for weights in (w, None):
        want, size = (torch.zeros(T, d, dtype=torch.float64, device=DEV) for _ in range(2))
        for j in range(k):
            term = Ys[at[:, j]].double() * (1.0 if weights is None else weights[:, j, None].double())
            term = torch.where(has[:, j, None], term, 0.0)
            want += term
            size += term.abs()
        for add in (False, "in place"):
            Y, buf, other = padded(T, d, dt, **style)
            if add:
                Y.copy_(a)
                want += a.double()
                size += a.double().abs()
            K.kfac_experts_combine(ctx.h, Ys, rows, weights, Y, add=Y if add else None)
            close(Y, want, (k + 2) * U * size + half_step(dt) * want.abs())
            assert bool((buf[other] == 5.0).all())
    del want, size, term
    G = padded(T, d, dt, **STYLES[(shape + 1) % 3])[0]
    G.copy_(g)
    dYs, buf, other = padded(R, d, dt, **style)
    dw = torch.full((T, k), math.nan, device=DEV)
    K.kfac_experts_combine_grad(ctx.h, G, Ys, rows, w, dYs, dw)
    for j in range(k):
        h = has[:, j]
        want = w[h, j, None].double() * g[h].double()
        close(dYs[at[h, j]], want, (U + half_step(dt)) * want.abs())
        term = g[h].double() * Ys[at[h, j]].double()
        close(dw[h, j], term.sum(1), (d + 2) * U * term.abs().sum(1))
        assert bool((dw[~h, j] == 0).all())
    assert bool((dYs[used:] == 5.0).all()) and bool((buf[other] == 5.0).all())


# more than 4096 slots, or more than 512 experts for over 2048: the copy adds up the order; rows of 1 to 513 vectors
RANKED = [(1500, 3, 40, 1), (1500, 3, 40, 3), (1500, 3, 40, 7), (4200, 1, 3, 8), (700, 6, 90, 66), (1500, 3, 40, 131), (2100, 2, 600, 264), (1500, 3, 40, 577), (700, 4, 600, 1031), (1500, 3, 40, 2049),
          (600, 8, 4096, 4099), (72, 64, 20, 520)]


@pytest.mark.parametrize("ws", [0, 8 << 20])
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("shape", range(len(RANKED)))
def test_copies_behind_a_sort_of_many(shape, bf16, ws):
    T, k, E, d = RANKED[shape]
    assert K.kfac_experts_dispatch_workspace_bytes(T, k, E) > 0
    dt, style = torch.bfloat16 if bf16 else torch.float32, STYLES[shape % 3]
    gen = torch.Generator().manual_seed(shape)
    c = Ctx(max(ws, 256))
    try:
        if ws == 0:
            K.kfac_destroy(c.h)
            c.h = K.kfac_create(0, c.stream.cuda_stream, None)
        x, ids, R = torch.randn(T, d, generator=gen).to(dt), random_ids(T, k, E, gen), T * k + shape % 4
        offsets, rows = torch.full((E + 1,), -7, dtype=torch.int32, device=DEV), torch.full((T, k), -7, dtype=torch.int32, device=DEV)
        Xs, buf, other = padded(R, d, dt, **style)
        K.kfac_experts_dispatch(c.h, ids.to(DEV), matrix(x, dt, **STYLES[(shape + 2) % 3])[0], offsets, rows, Xs)
        want_off, want_rows = order_of(ids, E)
        assert torch.equal(offsets.cpu(), want_off) and torch.equal(rows.cpu(), want_rows)
        has = want_rows >= 0
        want = torch.full((R, d), 5.0, dtype=dt)
        want[want_rows[has].long()] = x.repeat_interleave(k, 0)[has.view(-1)]
        assert torch.equal(Xs.cpu(), want) and bool((buf[other] == 5.0).all())
    finally:
        c.close()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("T,E,k", [(40, 2, 2), (50, 9, 9), (40, 16, 13), (33, 64, 8), (21, 40, 40), (9, 300, 64), (7, 1000, 64), (5, 3000, 3)])
def test_an_expert_more_than_once(ctx, T, E, k, bf16):
    """The gradient of the logits for ids that occur more than once, next to each other, apart and in all slots, and others that are nobody's."""
    dt = torch.bfloat16 if bf16 else torch.float32
    gen = torch.Generator().manual_seed(E + k)
    host = logits_for(T, E, "normal", gen).to(dt)
    x, dw = host.double(), torch.randn(T, k, generator=gen)
    given = choice(x, k)
    given[:, k // 2:] = given[:, :k - k // 2]
    given[1] = given[1, 0]
    given[2, -1] = given[2, 0]
    given[3] = torch.randint(-1, E + 1, (k,), generator=gen)
    given[4] = torch.randint(0, min(E, 3), (k,), generator=gen)
    for normalize in (False, True):
        out = torch.full((T, E), 5.0, dtype=dt, device=DEV)
        K.kfac_experts_route_grad(ctx.h, host.to(DEV), given.to(DEV), dw.to(DEV), out, normalize=normalize)
        ids = torch.where((given >= 0) & (given < E), given, -1)
        g, has, at = dw.double(), ids >= 0, ids.clamp(min=0).long()
        if normalize:
            p = weights_of(x, ids, True)
            d, size = p * (g - (p * g).sum(1, keepdim=True)), p * (g.abs() + (p * g.abs()).sum(1, keepdim=True))
            grad, size = (torch.zeros_like(x).scatter_add_(1, at, torch.where(has, v, 0.0)) for v in (d, size))
        else:
            p = softmax(x)
            at_e, size = (torch.zeros_like(x).scatter_add_(1, at, torch.where(has, v, 0.0)) for v in (g, g.abs()))
            grad, size = p * (at_e - (p * at_e).sum(1, keepdim=True)), p * (size + (p * size).sum(1, keepdim=True))
        # as for ids that differ: two softmaxes' errors, the sums' over experts and slots, and eight operations
        near(out, grad, (4 * (spread(x) + 8) + 2 * (E + 4) + k + 8) * U * size + half_step(dt) * grad.abs())


# ---------------------------------------------------------------- a launch has 2^23 workgroups at most
@pytest.fixture(autouse=True)
def memory_back(request):
    yield
    if "second_launch" in request.node.name:
        torch.cuda.empty_cache()


SECOND = 1 << 23


def test_copies_of_a_second_launch(ctx):
    """A token a workgroup: rows given, and rows behind a sort."""
    T, d, dt = SECOND + 3, 1032, torch.bfloat16
    X = torch.randn(1 << 20, d, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(dt).repeat(9, 1)[:T]
    X[SECOND:] = torch.arange(3 * d, device=DEV).view(3, d).to(dt)
    mine = torch.tensor([0, SECOND - 1, SECOND, SECOND + 2], device=DEV)
    rows = torch.full((T, 1), -1, dtype=torch.int32, device=DEV)
    rows[mine, 0] = torch.tensor([2, 0, 4, 3], dtype=torch.int32, device=DEV)
    Xs = torch.full((5, d), 3.0, dtype=dt, device=DEV)
    K.kfac_experts_gather(ctx.h, rows, X, Xs)
    assert torch.equal(Xs[[2, 0, 4, 3]], X[mine]) and bool((Xs[1] == 3.0).all())
    del Xs
    ids = torch.randint(-1, 3, (T, 1), dtype=torch.int32, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    offsets, Xs = torch.zeros(4, dtype=torch.int32, device=DEV), torch.empty(T, d, dtype=dt, device=DEV)
    K.kfac_experts_dispatch(ctx.h, ids, X, offsets, rows, Xs)
    order = torch.sort(torch.where(ids[:, 0] < 0, 3, ids[:, 0]), stable=True)[1]
    used = int((ids >= 0).sum())
    assert offsets.tolist() == [0] + [int((ids >= 0).logical_and(ids <= e).sum()) for e in range(3)]
    assert torch.equal(rows[order[:used], 0], torch.arange(used, dtype=torch.int32, device=DEV)) and bool((rows[order[used:]] == -1).all())
    for r in range(0, used, 1 << 20):
        assert torch.equal(Xs[r:min(r + (1 << 20), used)], X[order[r:min(r + (1 << 20), used)]])


def test_sums_of_a_second_launch(ctx):
    """A token a workgroup."""
    T, d = SECOND + 3, 2056
    v = torch.randn(2, d, generator=torch.Generator().manual_seed(0)).bfloat16().to(DEV)
    rows = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    rows[SECOND - 1], rows[SECOND], rows[-1] = 1, 1, -1
    Y = torch.full((T, d), 5.0, dtype=torch.bfloat16, device=DEV)
    K.kfac_experts_combine(ctx.h, v, rows, None, Y)
    for t, r in ((0, 0), (SECOND - 2, 0), (SECOND - 1, 1), (SECOND, 1), (SECOND + 1, 0)):
        assert torch.equal(Y[t], v[r])
    assert bool((Y[-1] == 0).all()) and bool((Y[:SECOND - 1, 7] == v[0, 7]).all()) and bool((Y[:SECOND - 1, -1] == v[0, -1]).all())


def test_gradients_of_sums_of_a_second_launch(ctx):
    T, d, dt = SECOND + 3, 1032, torch.bfloat16
    dY = torch.zeros(T, d, dtype=dt, device=DEV)
    mine = torch.tensor([0, SECOND - 1, SECOND, SECOND + 2], device=DEV)
    gen = torch.Generator().manual_seed(3)
    g, ys, w = torch.randn(4, d, generator=gen).to(dt).to(DEV), torch.randn(5, d, generator=gen).to(dt).to(DEV), torch.ones(T, 1, device=DEV)
    dY[mine], w[mine, 0] = g, torch.tensor([2.0, -0.5, 4.0, 1.0], device=DEV)       # (powers of two: products are exact)
    rows = torch.full((T, 1), -1, dtype=torch.int32, device=DEV)
    rows[mine, 0] = torch.tensor([2, 0, 4, 3], dtype=torch.int32, device=DEV)
    dYs, dw = torch.full((5, d), 3.0, dtype=dt, device=DEV), torch.full((T, 1), 9.0, device=DEV)
    K.kfac_experts_combine_grad(ctx.h, dY, ys, rows, w, dYs, dw)
    assert torch.equal(dYs[[2, 0, 4, 3]], (g.float() * w[mine]).to(dt)) and bool((dYs[1] == 3.0).all())
    term = g.double() * ys[[2, 0, 4, 3]].double()
    close(dw[mine, 0], term.sum(1), (d + 2) * U * term.abs().sum(1))
    assert int((dw != 0).sum()) == 4


def test_gradients_of_a_choice_of_a_second_launch(ctx):
    """Sixteen tokens a workgroup."""
    T, E = 16 * SECOND + 5, 17
    logits = torch.zeros(T, E, dtype=torch.bfloat16, device=DEV)
    ids, dw = torch.full((T, 1), 3, dtype=torch.int32, device=DEV), torch.ones(T, 1, device=DEV)
    ids[-2], dw[-1] = 16, -2.0
    out = torch.full((T, E), 5.0, dtype=torch.bfloat16, device=DEV)
    K.kfac_experts_route_grad(ctx.h, logits, ids, dw, out)
    p = 1.0 / E
    # (p is off by its sum's E + 2 roundings and two of its own)
    for part, chosen, size in ((slice(0, T - 2), 3, 1.0), (slice(T - 2, T - 1), 16, 1.0), (slice(T - 1, T), 3, -2.0)):
        for e in (0, 3, 8, 16):
            want = size * p * ((e == chosen) - p)
            assert float((out[part, e].float() - want).abs().max()) <= (half_step(torch.bfloat16) + 4 * (E + 8) * U) * abs(want)
