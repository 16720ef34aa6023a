"""A layer of experts through two whole training steps -- products, gradients, factors, eigendecomposition, preconditioning, AdamW -- against the
fp64 oracle and the formulas in float64, on the library's own parameters of each step."""
import numpy as np
import pytest
import torch

import oracle
from paper_2007_00784_amd.runner import ExpertRunner
from gpu_util import relfro

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16,bits", [(True, 8), (True, 32), (False, 32), (False, 8)])
def test_two_steps(bf16, bits):
    E, d_in, d_out, gamma = 4, 40, 24, 1e-3
    rng = np.random.default_rng(3)
    run = ExpertRunner(E, 403, d_in, d_out, bias=True, bf16=bf16, state_bits=bits, damping=gamma)
    dt = torch.bfloat16 if bf16 else torch.float32
    dev = run.dev
    run.load(torch.from_numpy(rng.normal(0, d_in ** -0.5, (E, d_out, d_in + 1)).astype(np.float32)))
    F = {k: np.zeros((E, n, n)) for k, n in (("A", d_in + 1), ("G", d_out))}
    m = v = np.zeros((E, d_out, d_in + 1))
    for step, counts in enumerate(([120, 80, 100, 100], [150, 0, 97, 153])):
        off = np.concatenate([[0], np.cumsum(counts)])
        offsets = torch.tensor(off, dtype=torch.int32, device=dev)
        x = torch.from_numpy(np.maximum(rng.normal(0, 1, (403, d_in)), 0).astype(np.float32)).to(dev).to(dt)
        g = torch.from_numpy(rng.normal(0, 0.1, (403, d_out)).astype(np.float32)).to(dev).to(dt)
        xs, gs = x.double().cpu().numpy(), g.double().cpu().numpy()
        W, P0 = run.weight.double().cpu().numpy(), run.param.double().cpu().numpy()
        y = run.forward(x, offsets).double().cpu().numpy()
        dx = run.backward(x, g, offsets).double().cpu().numpy()
        decay = 0.0 if step == 0 else 0.9
        run.update_factors(x, g, offsets, decay)
        run.eig()
        raw = run.grad.double().cpu().numpy()
        run.precondition()
        used = run.grad.double().cpu().numpy()
        clip = torch.tensor([0.5], device=dev)
        run.step(1e-2, grad_scale=clip)
        torch.cuda.synchronize()
        for e in range(E):
            r = slice(off[e], off[e + 1])
            n = counts[e]
            xt = np.concatenate([xs[r], np.ones((n, 1))], 1)
            if n:
                # one rounding to the type (2^-8 in bf16) and 41 or 24 additions in fp32, as norms
                tol = 2.0 ** -8 + 1e-6 if bf16 else 2e-5
                assert relfro(y[r], xt @ W[e].T) <= tol and relfro(dx[r], gs[r] @ W[e, :, :d_in]) <= tol
                assert relfro(raw[e], gs[r].T @ xt) <= 2e-5
                F["A"][e] = decay * F["A"][e] + (1 - decay) * oracle.gram(xs[r], 1, 1.0 / n)
                F["G"][e] = decay * F["G"][e] + (1 - decay) * oracle.gram(gs[r], 0, 1.0 / n)
            else:
                assert not raw[e].any()
            assert relfro(run.A[e].double().cpu().numpy(), F["A"][e]) <= 2e-5 and relfro(run.G[e].double().cpu().numpy(), F["G"][e]) <= 2e-5
            la, qa = oracle.eigh(F["A"][e])
            lg, qg = oracle.eigh(F["G"][e])
            if n:
                assert relfro(used[e], oracle.precondition(qa, la, qg, lg, gamma, raw[e])) <= 1e-4     # the bound of the preconditioner's own tests
            else:
                assert not used[e].any()
        # the optimizer step on what the preconditioner left
        if bits == 8 and step == 1:
            m, v = values["m"], values["v"] ** 2
        m = 0.9 * m + 0.1 * 0.5 * used
        v = 0.999 * v + 0.001 * (0.5 * used) ** 2
        t = step + 1
        upd = (m / (1 - 0.9 ** t)) / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
        want = P0 - 1e-2 * 0.01 * P0 - 1e-2 * upd
        got = run.param.double().cpu().numpy()
        # fp32: a dozen roundings of an update of size 1e-2 * (at most 3 here), the parameter's own roundings
        assert (np.abs(got - want) <= 2.0 ** -22 * np.abs(P0) + 1e-2 * 32 * 2.0 ** -24 * (1 + np.abs(upd))).all()
        if bf16:
            assert torch.equal(run.weight, run.param.to(torch.bfloat16))
        if bits == 8:
            from paper_2007_00784_amd import kfac as K
            values = {}
            for k, ref in (("m", m), ("v", np.sqrt(v))):
                out = torch.empty(m.size, device=dev)
                K.kfac_adamw_state_values(run.ctx, run.state[k], run.state[k + "_scale"], out)
                values[k] = out.double().cpu().numpy().reshape(m.shape)
                # half a step of e4m3 is 2^-4 of the value, and 2^-10 of a scale of at most the largest / 224 below
                block = np.abs(ref).reshape(-1)
                big = np.array([block[i // 128 * 128:i // 128 * 128 + 128].max() for i in range(0, len(block), 128)]).repeat(128)[:len(block)].reshape(ref.shape)
                small = 2.0 ** -9 * big / 224 if k == "v" else 2.0 ** -10 * big / 224
                assert (np.abs(values[k] - ref) <= (2.0 ** -4 + 1e-5) * np.abs(ref) + small).all()
        else:
            assert relfro(run.state["m"].cpu().numpy().reshape(m.shape), m) <= 2e-6 and relfro(run.state["v"].cpu().numpy().reshape(m.shape), v) <= 2e-6
    run.close()
