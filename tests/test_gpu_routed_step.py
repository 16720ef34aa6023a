"""A layer of experts behind its router through two training steps -- choice, sort, products, weighted sum, all gradients, preconditioning, clipping,
AdamW -- against autograd in float64 on the library's own parameters and choices of each step."""
import math

import pytest
import torch

from paper_2007_00784_amd.runner import ExpertRunner, KfacRunner, RoutedExpertRunner
from paper_2007_00784_amd import synthetic as S
from gpu_util import relfro

pytestmark = pytest.mark.gpu


def reference(run, x, g, add):
    """Output and gradients (tokens, experts' weights, router) by autograd in float64, with the run's ids."""
    f = lambda t: t.detach().double().cpu()  # noqa: E731
    X, W, Wr = f(x).requires_grad_(), f(run.weight).requires_grad_(), f(run.router_weight)[0].requires_grad_()
    ids = run.ids.cpu().long()
    d = X.shape[1]
    logits = X @ Wr.t()
    w = torch.gather(torch.softmax(logits, 1), 1, ids)
    if run.normalize:
        w = w / w.sum(1, keepdim=True)
    pick = W[ids]                                                        # [T, k, d_out, d + 1]
    y = (pick[..., :d] * X[:, None, None, :]).sum(3) + (pick[..., d] if run.bias else 0.0)
    out = (y * w[:, :, None]).sum(1)
    if add is not None:
        out = out + f(add)
    out.backward(f(g))
    return [t.detach() for t in (logits, out, X.grad, W.grad, Wr.grad)]


@pytest.mark.parametrize("bf16,bits,normalize,T,k", [(True, 8, True, 200, 2), (True, 32, False, 700, 3), (False, 32, True, 700, 3), (False, 8, False, 33, 1)])
def test_two_steps(bf16, bits, normalize, T, k):
    E, d_in, d_out, lr = 5, 48, 40, 1e-2
    gen = torch.Generator().manual_seed(7)
    run = RoutedExpertRunner(E, T, k, d_in, d_out, normalize=normalize, bf16=bf16, state_bits=bits)
    rand = lambda *s, scale=1.0: torch.randn(*s, generator=gen) * scale  # noqa: E731
    run.load(rand(E, d_out, d_in + 1, scale=d_in ** -0.5), rand(1, E, d_in, scale=d_in ** -0.5))
    moments = None
    for step in range(2):
        x, g, add = (rand(T, n).to(run.dt).to(run.dev) for n in (d_in, d_out, d_out))
        if step == 0:
            add = None
        y = run.forward(x, add).clone()
        dx = run.backward(x, g).clone()
        ref = reference(run, x, g, add)
        # fp32: sums of some ten thousand products at most.  bf16: logits, rows, their results and gradients are rounded one after another, each by 2^-9 on
        # average and 2^-8 at most, and a logit's rounding moves its weight by as much: a path has at most eight of them
        tol = 8 * 2.0 ** -8 if bf16 else 2e-5
        for name, got, want in zip(("logits", "out", "tokens", "experts", "router"), (run.logits, y, dx, run.grad, run.router_grad[0]), ref):
            assert relfro(got.double().cpu(), want) <= tol, name
        # the choice is that of the logits
        left = run.logits.double().cpu()
        assert torch.equal(run.ids.cpu().long(), torch.sort(left, dim=1, descending=True, stable=True)[1][:, :k])
        run.update_factors(0.0 if step == 0 else 0.9)
        run.eig()
        run.precondition()
        grads = [run.grad.double().cpu(), run.router_grad.double().cpu()]
        want = math.sqrt(sum(float((t ** 2).sum()) for t in grads))
        before = [run.param.double().cpu(), run.router.double().cpu()]
        coef = run.clip(want / 3)
        run.step(lr, grad_scale=coef)
        torch.cuda.synchronize()
        assert abs(float(run.norm) - want) <= 1e-6 * want and abs(float(coef) - 1 / 3) <= 1e-6
        if bits == 32:
            c = [t / 3 for t in grads]
            moments = [(0.1 * t, 0.001 * t * t) if moments is None else (0.9 * m + 0.1 * t, 0.999 * v + 0.001 * t * t) for t, (m, v) in zip(c, moments or [(0, 0)] * 2)]
            for p, b, (m, v) in zip((run.param, run.router), before, moments):
                t = step + 1
                upd = (m / (1 - 0.9 ** t)) / (torch.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
                # (the coefficient's 1e-6 counts beside eps only; a dozen roundings of an update of up to 3)
                assert ((p.double().cpu() - (b - lr * 0.01 * b - lr * upd)).abs() <= 2.0 ** -22 * b.abs() + lr * (2e-6 + 64 * 2.0 ** -24) * (1 + upd.abs())).all()
        if bf16:
            assert torch.equal(run.weight, run.param.to(run.dt)) and torch.equal(run.router_weight, run.router.to(run.dt))
    run.close()


def test_accumulated_batches():
    """Two batches before one step: gradients add up, the tokens' do not."""
    run = RoutedExpertRunner(3, 50, 2, 24, 16, bf16=False)
    gen = torch.Generator().manual_seed(1)
    run.load(torch.randn(3, 16, 25, generator=gen) * 0.2, torch.randn(1, 3, 24, generator=gen) * 0.2)
    sums = [torch.zeros_like(run.grad), torch.zeros_like(run.router_grad)]
    batches = [(torch.randn(50, 24, generator=gen).to(run.dev), torch.randn(50, 16, generator=gen).to(run.dev)) for _ in range(2)]
    alone = []
    for x, g in batches:
        run.forward(x)
        alone.append(run.backward(x, g).clone())
        for s, t in zip(sums, (run.grad, run.router_grad)):
            s += t
    for i, (x, g) in enumerate(batches):
        run.forward(x)
        run.xs.fill_(float("nan"))                           # another layer's by now
        assert torch.equal(run.backward(x, g, accumulate=i > 0, gather=True), alone[i])
    for s, t in zip(sums, (run.grad, run.router_grad)):
        assert relfro(t.double().cpu(), s.double().cpu()) <= 1e-6
    run.close()


def test_padding_and_experts_out_of_use():
    """Padded tokens get what is added and no gradients; an expert out of use no rows; the others are those of a batch without either."""
    T, E, live = 60, 5, 41
    gen = torch.Generator().manual_seed(3)
    W, Wr = torch.randn(E, 16, 25, generator=gen) * 0.2, torch.randn(1, E, 24, generator=gen) * 0.2
    x, g, add = torch.randn(T, 24, generator=gen), torch.randn(T, 16, generator=gen), torch.randn(T, 16, generator=gen)
    masked = torch.zeros(T, E, dtype=torch.bool)
    masked[live:] = True
    masked[:, 2] = True
    results = []
    for n in (T, live):
        run = RoutedExpertRunner(E, n, 2, 24, 16, bf16=False)
        run.load(W, Wr)
        dev = lambda t: t[:n].to(run.dev)  # noqa: E731
        y = run.forward(dev(x), dev(add), masked=dev(masked))
        if n == T:
            assert torch.equal(y[live:], dev(add)[live:]) and (run.ids[live:] == -1).all() and (run.row[live:] == -1).all()
        assert int(run.offsets[2]) == int(run.offsets[3]) and int(run.offsets[-1]) == 2 * live
        dx = run.backward(dev(x), dev(g))
        assert (dx[live:] == 0).all() and not run.grad[2].any() and not run.router_grad[0, 2].any()
        results.append([t.clone() for t in (y[:live], dx[:live], run.grad, run.router_grad)])
        run.close()
    for a, b in zip(*results):                               # (sums over more rows may go in other parts)
        assert relfro(a.double().cpu(), b.double().cpu()) <= 1e-6


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("whole", [True, False])
def test_padding_that_holds_anything(whole, bf16):
    """What stands in padded tokens, NaN and infinities among it, and in their outputs' gradients reaches nothing: the same bits as with zeros there."""
    T, E, k, live = 70, 5, 2, 53
    gen = torch.Generator().manual_seed(11)
    W, Wr = torch.randn(E, 16, 25, generator=gen) * 0.2, torch.randn(1, E, 24, generator=gen) * 0.2
    batches = [(torch.randn(T, 24, generator=gen), torch.randn(T, 16, generator=gen)) for _ in range(2)]
    masked = torch.zeros(T, 1 if whole else E, dtype=torch.bool)
    masked[live:] = True
    masked[7] = True
    pad = masked[:, 0].clone()
    if not whole:
        masked[:, 3] = True
    results = []
    for odd in (torch.tensor([0.0]), torch.tensor([math.nan, math.inf, -math.inf, 1e30])):
        run = RoutedExpertRunner(E, T, k, 24, 16, bf16=bf16)
        run.load(W, Wr)
        out = []
        for i, batch in enumerate(batches):
            x, g = (t.clone() for t in batch)
            for t in (x, g):
                t[pad] = odd[torch.arange(int(pad.sum()) * t.shape[1]) % odd.numel()].view(-1, t.shape[1])
            x, g = x.to(run.dt).to(run.dev), g.to(run.dt).to(run.dev)
            kept = x.clone()
            out.append(run.forward(x, masked=masked.to(run.dev)).clone())
            out.append(run.backward(x, g, accumulate=i > 0, gather=i > 0).clone())
            assert torch.equal(x.view(torch.int16), kept.view(torch.int16))
        run.update_factors(0.5)
        results.append(out + [t.clone() for t in (run.grad, run.router_grad, run.A, run.G)])
        run.close()
    for a, b in zip(*results):
        assert a.isfinite().all() and torch.equal(a, b)


def test_clip_of_other_runners():
    """The gradients of a network in place, and the coefficient of a layer of experts."""
    run = KfacRunner(S.workload("resnet32_cifar"), n_updates=1, batch=2, layers=[0, 3, 33])
    run.restore_gradients()
    raw = [g.double().cpu() for g in run.grad]
    want = math.sqrt(sum(float((g ** 2).sum()) for g in raw))
    run.clip(want / 2)
    for g, r in zip(run.grad, raw):
        assert relfro(g.double().cpu(), r / 2) <= 1e-6
    assert abs(float(run.norm) - want) <= 1e-6 * want
    run.clip(want)
    assert float(run.coef) == 1.0
    run.close()
    run = ExpertRunner(2, 10, 8, 8)
    run.grad.fill_(2.0)
    n = math.sqrt(run.grad.numel() * 4.0)
    assert abs(float(run.clip(n / 4, grad_scale=torch.full((1,), 0.5, device=run.dev))) - 0.25) <= 1e-6 and abs(float(run.norm) - n / 2) <= 1e-6 * n
    run.close()


def busy(n=12):
    """Some milliseconds of work for the current stream."""
    a = torch.zeros(8192, 8192, dtype=torch.bfloat16, device="cuda:0")
    for _ in range(n):
        a = a @ a


@pytest.mark.parametrize("before", ["runner", "caller", "neither"])
@pytest.mark.parametrize("same", [True, False])
def test_on_its_own_stream(same, before):
    """A runner made on a side stream and called from it, or from another one, either of them busy: parameters, masks and padding take effect in the order of the calls."""
    T, E, k = 300, 6, 2
    gen = torch.Generator().manual_seed(5)
    params = [(torch.randn(E, 16, 25, generator=gen) * 0.2, torch.randn(1, E, 24, generator=gen) * 0.2) for _ in range(2)]
    x, g = torch.randn(T, 24, generator=gen).cuda(), torch.randn(T, 16, generator=gen).cuda()
    x[250:] = math.nan
    lengths = torch.tensor([250], device="cuda:0")
    out = torch.tensor([[False, True, False, False, False, False]], device="cuda:0")
    torch.cuda.synchronize()
    results = []
    for side in (None, torch.cuda.Stream()):
        with torch.cuda.stream(side or torch.cuda.current_stream()):
            run = RoutedExpertRunner(E, T, k, 24, 16, bf16=True)
        xs, gs = x.to(run.dt), g.to(run.dt)
        device = [[t.cuda() for t in p] for p in params]
        torch.cuda.synchronize()
        with torch.cuda.stream(side if side is not None and same else torch.cuda.current_stream()):
            for p in device:
                if side is not None and before != "neither":
                    with torch.cuda.stream(side if before == "runner" else torch.cuda.current_stream()):
                        busy()
                run.load(*p)
                masked = (torch.arange(T, device="cuda:0") >= lengths)[:, None] | out
                run.forward(xs, masked=masked)
                del masked
                torch.ones(T, E, dtype=torch.bool, device="cuda:0")       # (takes the memory of the mask)
                run.backward(xs, gs)
        torch.cuda.synchronize()
        assert (run.ids[250:] == -1).all() and not (run.ids == 1).any() and int(run.offsets[-1]) == 250 * k
        results.append([t.clone() for t in (run.out, run.dtokens, run.grad, run.router_grad)])
        run.close()
    for a, b in zip(*results):
        assert a.isfinite().all() and torch.equal(a, b)


def test_clip_from_a_busy_stream():
    """Gradients are restored and clipped for the first time from a busy stream that is not the runner's: none of it comes behind what it has to precede."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run = KfacRunner(S.workload("resnet32_cifar"), n_updates=1, batch=2, layers=[0, 3, 33])
    torch.cuda.synchronize()
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in run.gradw_master))
    torch.cuda.synchronize()
    busy()
    run.restore_gradients()
    run.clip(want / 2)
    torch.cuda.synchronize()
    assert abs(float(run.norm) - want) <= 1e-6 * want and abs(float(run.coef) - 0.5) <= 1e-6
    for g, r in zip(run.grad, run.gradw_master):
        assert relfro(g.double().cpu(), r.double().cpu() / 2) <= 1e-6
    run.close()


@pytest.mark.parametrize("bf16", [True, False])
def test_captured_with_masks(bf16):
    """A masked batch forth and back and its norm as a graph: every replay, with eager work between them, gives the bits of an eager run of the same inputs."""
    T, E, k = 90, 5, 2
    gen = torch.Generator().manual_seed(2)
    W, Wr = torch.randn(E, 16, 25, generator=gen) * 0.2, torch.randn(1, E, 24, generator=gen) * 0.2
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run = RoutedExpertRunner(E, T, k, 24, 16, bf16=bf16)
    eager = RoutedExpertRunner(E, T, k, 24, 16, bf16=bf16)
    for r in (run, eager):
        r.load(W, Wr)
    x, g, masked = (torch.zeros(T, n, dtype=dt, device=run.dev) for n, dt in ((24, run.dt), (16, run.dt), (E, torch.bool)))

    def step(r):
        y = r.forward(x, masked=masked)
        return y, r.backward(x, g), r.grad, r.router_grad, r.clip(0.5), r.norm

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(run)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outputs = step(run)
    for seed in (1, 2, 3):
        gen = torch.Generator().manual_seed(seed)
        pad = torch.rand(T, 1, generator=gen) < 0.2
        x.copy_(torch.where(pad, math.nan, torch.randn(T, 24, generator=gen)))
        g.copy_(torch.randn(T, 16, generator=gen))
        masked.copy_(pad | (torch.rand(1, E, generator=gen) < 0.3))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs, step(eager)):
            assert a.isfinite().all() and torch.equal(a, b)
        torch.cuda.synchronize()
    run.close()
    eager.close()
