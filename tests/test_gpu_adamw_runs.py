"""AdamW with 8-bit state over whole runs, against moments in float64 that are never rounded to codes.

Bounds.  A code is drawn so that its expectation is the value, hence that of m is the formula's.  sqrt(v) goes on as sqrt(beta2 r^2 + (1 - beta2) g^2),
which is convex in the held root r: its expectation is not below the formula's.  Above: a step of size d between codes D <= r / 8 apart has a
variance of d D at most, which is added to v.  With d <= (1 - beta2) / 2 |g^2 / r^2 - 1| r (0.97 in the mean for normal g) that is (1 - beta2) 6 % of v a
step, so 6 % of v and 3 % of the root where gradients stay as they are; where v decays by a hundredth (4.6 / (1 - beta2) steps) it is exp(4.6 / 16) = 1.33
of v, 1.16 of the root.  Sampling: the same variances leave a root off by 17 % (standard deviation) from its expectation; the mean of 8192 by 0.2 %.
"""
import numpy as np
import pytest
import torch

from paper_2007_00784_amd import kfac as K
from paper_2007_00784_amd.runner import ExpertRunner
from gpu_util import Ctx
from test_gpu_adamw import BLOCK, HYPER, Tensor, adam64, block_scales, codes_of_e4m3

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SAMPLING = 0.01      # of a mean of 8192, five standard deviations


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(1 << 20)
    yield c
    c.close()


def eight(n):
    blocks = (n + BLOCK - 1) // BLOCK
    z = lambda k, dt: torch.zeros(k, dtype=dt, device=DEV)  # noqa: E731
    return dict(param=z(n, torch.float32), grad=z(n, torch.float32), m=z(n, torch.uint8), v=z(n, torch.uint8), m_scale=z(blocks, torch.uint8), v_scale=z(blocks, torch.uint8))


def held(h, t, k):
    out = torch.empty(t["param"].numel(), device=DEV)
    K.kfac_adamw_state_values(h, t[k], t[k + "_scale"], out)
    return out.double()


STEADY, DECAYING = 1.03 + SAMPLING, 1.16 + SAMPLING
# beta2, gradients, the step from which they are a tenth, steps, at most (of the mean root)
RUNS = [(0.999, "normal", None, 2000, STEADY), (0.95, "normal", None, 2000, STEADY), (0.999, "constant", None, 2000, STEADY), (0.999, "normal", 1000, 6000, DECAYING),
        (0.95, "normal", 1000, 2000, STEADY), (0.999, "normal", None, 100, STEADY)]


@pytest.mark.parametrize("run", range(len(RUNS)))
def test_state_follows_its_moments(ctx, run):
    b2, kind, drop, steps, most = RUNS[run]
    n, b1 = 8192, 0.9
    gen = torch.Generator(DEV).manual_seed(run)
    t = eight(n)
    items = K.adamw_items([t])
    m, v = (torch.zeros(n, dtype=torch.float64, device=DEV) for _ in range(2))
    for k in range(1, steps + 1):
        if kind == "normal":
            t["grad"].normal_(generator=gen)
        else:
            t["grad"].fill_(1.0)
        if drop is not None and k > drop:
            t["grad"].mul_(0.1)
        g = t["grad"].double()
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        t["param"].zero_()
        K.kfac_adamw_batched(ctx.h, items, lr=1.0, beta1=b1, beta2=b2, weight_decay=0.0, step=k, seed=99)
    root = held(ctx.h, t, "v").mean() / v.sqrt().mean()
    assert 1 - SAMPLING <= float(root) <= most
    # a code of m is off by a sixteenth of it at most as a standard deviation, the average of 1 / (1 - beta1^2) such by a seventh; over 8192 elements
    # five of them are 1 %
    slope = (held(ctx.h, t, "m") * m).sum() / (m * m).sum()
    assert abs(float(slope) - 1) <= 0.01
    if most == STEADY:
        # the update: (1 / 7)^2 of m^2 is 1 % of its root, 17 % of the root of v 4.4 % of the root of the mean 1 / v, less the 3 % above
        want = (m / (1 - b1 ** steps)) / ((v / (1 - b2 ** steps)).sqrt() + 1e-8)
        assert 0.96 <= float((t["param"].double().square().mean() / want.square().mean()).sqrt()) <= 1.06


def test_a_code_is_one_of_the_two_around_the_value(ctx):
    """And the upper one with the probability of the distance from the lower: the errors of a step, in distances of codes, have a mean of zero."""
    n = 20011
    t = Tensor(n, 8, seed=3)
    K.kfac_adamw_batched(ctx.h, [t.t], step=3, seed=7, **HYPER)
    torch.cuda.synchronize()
    w = t.was
    _, m, v, _ = adam64(w["param"], w["grad"], w["m"], w["v"], 3, HYPER)
    for k, x, err, least in (("m", m, 4 * 2.0 ** -24 * (np.abs(w["m"]) + np.abs(w["grad"])), 0.0), ("v", np.sqrt(v), 5 * 2.0 ** -24 * np.sqrt(v), 2.0 ** -9)):
        s = t.t[k + "_scale"].cpu().numpy().astype(int) - 127
        assert (np.abs(s - block_scales(x)) <= 1).all()
        unit = 2.0 ** np.repeat(s, BLOCK)[:n]
        y = np.abs(x) / unit
        y = np.where(y > 0, np.maximum(y, least), y)
        apart = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
        off = (np.abs(t.values(k)) / unit - y) / apart
        # (a value within its error of a code can be that code's neighbour below or above)
        assert (np.abs(off) <= 1 + 2 * err / unit / apart).all()
        assert (np.abs(off) > 0.5).any()
        inside = (y >= 2.0 ** -9) & (y < 440)
        assert abs(off[inside].mean()) <= 5 * 0.5 / np.sqrt(inside.sum())
        assert ((np.sign(t.values(k)) == np.sign(x)) | (t.values(k) == 0)).all()
        assert k == "m" or (t.values(k)[x > 0] > 0).all()


def test_what_is_drawn_follows_from_seed_step_and_place(ctx):
    n = 3000
    make = lambda: [Tensor(n, 8, seed=5, copy=True).t for _ in range(2)]  # noqa: E731
    runs = []
    for step, seed in ((3, 7), (3, 7), (3, 8), (3, 7 + (1 << 40)), (4, 7)):
        ts = make()
        K.kfac_adamw_batched(ctx.h, ts, step=step, seed=seed, **HYPER)
        runs.append(ts)
    torch.cuda.synchronize()
    first = runs[0]
    for a, b in zip(first, runs[1]):
        assert all(torch.equal(a[k], b[k]) for k in a)
    for other in runs[2:]:
        for k in ("m", "v"):
            assert not torch.equal(first[0][k], other[0][k])
    assert not torch.equal(first[0]["m"], first[1]["m"]) and not torch.equal(first[0]["v"], first[1]["v"])
    for other in runs[2:4]:      # the parameter goes with the moments before they are rounded
        assert torch.equal(first[0]["param"], other[0]["param"])


def test_long_lists_and_both_kinds_of_state(ctx):
    """The same tensor at many places of a list longer than a launch: each place draws words of its own, and tensors in 32 bits do not count."""
    ts = [Tensor(700, 8, seed=1).t for _ in range(120)]
    K.kfac_adamw_batched(ctx.h, ts, step=3, seed=7, **HYPER)
    codes = torch.stack([t["v"] for t in ts]).cpu().numpy()
    assert len({c.tobytes() for c in codes}) == 120
    again = [Tensor(700, 8, seed=1).t for _ in range(120)]
    mixed = [x for t in again for x in (Tensor(50, 32, seed=2).t, t)]
    K.kfac_adamw_batched(ctx.h, mixed, step=3, seed=7, **HYPER)
    assert all(torch.equal(a[k], b[k]) for a, b in zip(ts, again) for k in a)


def test_zero_and_what_is_not_finite(ctx):
    """A state of zero stays one, a gradient of zero adds nothing, NaN stays with its element, and behind a tensor's end nothing is written."""
    t = Tensor(300, 8)
    for k in t.t:
        if k != "param":
            t.t[k].zero_()
    K.kfac_adamw_batched(ctx.h, [t.t], step=1, seed=3, **HYPER)
    assert not any(bool(t.t[k].any()) for k in ("m", "v", "m_scale", "v_scale"))
    t = Tensor(131, 8)
    bufs = {k: x._base.clone() for k, x in t.t.items()}
    t.t["grad"][[3, 130]] = torch.tensor([float("nan"), float("inf")], device=DEV)
    K.kfac_adamw_batched(ctx.h, [t.t], step=3, seed=3, **HYPER)
    bad = (t.t["m"] & 127) == 127
    assert bad.nonzero().flatten().tolist() == [3, 130] and torch.equal(bad, (t.t["v"] & 127) == 127)
    assert (~torch.isfinite(t.t["param"])).nonzero().flatten().tolist() == [3, 130]
    for k, x in t.t.items():
        assert torch.equal(x._base[len(x):].view(torch.uint8), bufs[k][len(x):].view(torch.uint8)), k


def test_captured_with_the_step_on_the_gpu():
    """Each replay draws what the eager call of that step does."""
    s = torch.cuda.Stream()
    h = K.kfac_create(0, s.cuda_stream, None)
    eager = K.kfac_create(0, torch.cuda.current_stream().cuda_stream, None)
    a, b = Tensor(4097, 8, seed=5), Tensor(4097, 8, seed=5)
    step = torch.tensor([0], dtype=torch.int64, device=DEV)
    items = K.adamw_items([a.t])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step.add_(1)
        K.kfac_adamw_batched(h, items, step=step, seed=1 << 63, **HYPER)
    step.zero_()
    for k in range(1, 6):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        K.kfac_adamw_batched(eager, [b.t], step=k, seed=1 << 63, **HYPER)
        torch.cuda.synchronize()
        assert all(torch.equal(a.t[x], b.t[x]) for x in a.t), k
    K.kfac_destroy(h)
    K.kfac_destroy(eager)


def test_the_runner_of_a_layer_of_experts_follows():
    """300 steps of ExpertRunner with 8-bit state, the first of them rounded to nearest."""
    run = ExpertRunner(8, 16, 63, 64, bias=True, bf16=True, state_bits=8)
    gen = torch.Generator(DEV).manual_seed(4)
    v = torch.zeros(run.grad.numel(), dtype=torch.float64, device=DEV)
    for _ in range(300):
        run.grad.normal_(generator=gen)
        v = 0.999 * v + 0.001 * run.grad.double().flatten() ** 2
        run.step(1e-4)
    out = torch.empty(v.numel(), device=DEV)
    K.kfac_adamw_state_values(run.ctx, run.state["v"], run.state["v_scale"], out)
    # (the steps to nearest leave 1 / 16 at most of a share of 8 / 300)
    assert 1 - SAMPLING <= float(out.double().mean() / v.sqrt().mean()) <= STEADY
    assert run.steps == 300
    run.close()


@pytest.mark.parametrize("seed", [0, 5])
def test_roots_that_have_no_square_in_fp32(ctx, seed):
    """Gradients and roots from 2^-100 to 2^100, block by block: a root is lost neither below 2^-75 nor from 2^64 on, where v is 0 or infinite in fp32."""
    n = 201 * BLOCK
    size = 2.0 ** np.repeat(np.arange(-100, 101), BLOCK)
    t = Tensor(n, 8, seed=11)
    for k in ("m_scale", "v_scale"):
        t.t[k].copy_(torch.arange(-100, 101) + 127 - 8)
    g = np.random.default_rng(12).normal(0, 1, n) * size
    g[::3] = 0.0                                             # (what is held goes on by itself)
    t.t["grad"].copy_(torch.from_numpy(g))
    t.was["grad"] = t.t["grad"].cpu().double().numpy()
    t.was["m"], t.was["u"] = t.values("m"), t.values("v")
    t.was["v"] = t.was["u"] ** 2
    K.kfac_adamw_batched(ctx.h, [t.t], step=3, seed=seed, **HYPER)
    torch.cuda.synchronize()
    if seed == 0:
        t.check()
    _, m, v, upd = adam64(*(t.was[k] for k in ("param", "grad", "m", "v")), 3, HYPER)
    assert (np.isfinite(t.values("m")) & np.isfinite(t.values("v"))).all() and (t.values("v")[v > 0] > 0).all()
    # between neighbouring codes: an eighth of the value, or 2^-9 of the block's unit, whose 448 are at most twice its largest
    big = np.repeat(np.sqrt(v).reshape(-1, BLOCK).max(1), BLOCK)
    assert (np.abs(t.values("v") - np.sqrt(v)) <= (1 / 8 + 1e-6) * np.sqrt(v) + 2.0 ** -9 * big / 224).all()
    assert np.isfinite(t.t["param"].cpu().numpy()).all()


@pytest.mark.parametrize("seed", [0, 5])
def test_moments_at_the_end_of_the_range(ctx, seed):
    """Gradients of fp32's largest number for many steps: m and sqrt(v) stay finite, and are held as 448 * 2^119 at most."""
    t = eight(256)
    t["grad"].fill_(torch.finfo(torch.float32).max)
    t["grad"][128:] *= -0.9
    for step in range(1, 6):
        K.kfac_adamw_batched(ctx.h, [t], lr=1e-3, beta1=0.0, beta2=0.0, step=step, seed=seed)
        assert bool(torch.isfinite(t["param"]).all())
        for k in ("m", "v"):
            assert held(ctx.h, t, k).abs().tolist() == [448 * 2.0 ** 119] * 256 and t[k + "_scale"].tolist() == [246, 246]
        assert bool((held(ctx.h, t, "m")[128:] < 0).all())


def test_values_of_the_smallest_and_largest_scales(ctx):
    """Every code with the scales 0 to 4 and 243 to 247: exact in fp32, in bf16 from scale 3 on and the nearest number below.  No step leaves 247: its
    codes from 256 on are 2^128 and more, above fp32's (and bf16's) largest number."""
    table = codes_of_e4m3()
    for scale in (0, 1, 2, 3, 4, 243, 247):
        codes = torch.arange(256, dtype=torch.uint8, device=DEV)
        codes[(codes & 127) == 127] = 0
        scales = torch.full((2,), scale, dtype=torch.uint8, device=DEV)
        c = codes.cpu().numpy().astype(int)
        want = torch.from_numpy(np.where(c >= 128, -1.0, 1.0) * table[c & 127] * 2.0 ** (scale - 127))
        for dt in (torch.float32, torch.bfloat16):
            out = torch.empty(256, dtype=dt, device=DEV)
            K.kfac_adamw_state_values(ctx.h, codes, scales, out)
            # (float64 to float32 is exact here, float32 to bfloat16 rounds half to even)
            assert torch.equal(out.cpu().double(), want.float().to(dt).double()), (scale, dt)
            there = want.abs() < 2.0 ** 128
            assert bool(there.all()) == (scale <= 246)
            assert scale < 3 or torch.equal(out.cpu().double()[there], want[there])


def test_a_large_root_that_does_not_count(ctx):
    """beta2 = 0: the root is the gradient's size, however large the last one was."""
    t = eight(256)
    t["v"].fill_(0x38)                                       # 1
    t["v_scale"].fill_(127 + 60)
    t["grad"].fill_(-2.0 ** -20)
    K.kfac_adamw_batched(ctx.h, [t], lr=1e-3, beta2=0.0, step=2)
    assert held(ctx.h, t, "v").tolist() == [2.0 ** -20] * 256
