"""Layers of experts and AdamW on tensors with elements beyond 2^31: what is computed there is bit for bit what the same call gives on a short copy."""
import pytest
import torch

from paper_2007_00784_amd import kfac as K
from gpu_util import Ctx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(64 << 20)
    yield c
    c.close()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_the_largest_pitch(ctx, bf16):
    """2100 rows of 72 and 40 elements with 2^20 from one to the next."""
    dt, pitch, R, d_in, d_out = torch.bfloat16 if bf16 else torch.float32, 1 << 20, 2100, 72, 40
    gen = torch.Generator(DEV).manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dt)
    offsets = torch.tensor([3, 40, 40, 2000, 2095], dtype=torch.int32, device=DEV)
    far = lambda d: torch.empty(R * pitch, dtype=dt, device=DEV).as_strided((R, d), (pitch, 1))
    X, G, W = rand(R, d_in), rand(R, d_out), rand(4, d_out, d_in)
    fX, fG = far(d_in), far(d_out)
    fX.copy_(X)
    fG.copy_(G)
    out = far(d_in)
    for call, a, fa, width in ((K.kfac_experts_forward, X, fX, d_out), (K.kfac_experts_input_grad, G, fG, d_in)):
        short, far_out = torch.zeros(R, width, dtype=dt, device=DEV), out[:, :width]
        far_out.zero_()
        call(ctx.h, a, W, offsets, short)
        call(ctx.h, fa, W, offsets, far_out)
        assert torch.equal(far_out, short) and float(short[2094].abs().max()) > 0 and float(short[2095:].abs().max()) == 0
    dW, fdW = (torch.zeros(4, d_out, d_in, device=DEV) for _ in range(2))
    K.kfac_experts_weight_grad(ctx.h, G, X, offsets, dW)
    K.kfac_experts_weight_grad(ctx.h, fG, fX, offsets, fdW)
    assert torch.equal(dW, fdW) and float(dW[3].abs().max()) > 0
    F, fF = (torch.zeros(4, d_in, d_in, device=DEV) for _ in range(2))
    K.kfac_update_factors_experts(ctx.h, X, offsets, F)
    K.kfac_update_factors_experts(ctx.h, fX, offsets, fF)
    assert torch.equal(F, fF) and float(F[3].abs().max()) > 0


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_weights_beyond_31_bits(ctx, bf16):
    """700 experts of 1801 x 1800, of which the first and the last have rows: the last one's weights and gradient begin behind 2^31 elements."""
    dt, E, d_in, d_out, R = torch.bfloat16 if bf16 else torch.float32, 700, 1800, 1801, 37
    gen = torch.Generator(DEV).manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dt)
    assert (E - 1) * d_in * d_out > 1 << 31
    W = torch.zeros(E, d_out, d_in, dtype=dt, device=DEV)
    W[0], W[-1] = rand(d_out, d_in), rand(d_out, d_in)
    X, G = rand(R, d_in), rand(R, d_out)
    offsets = torch.full((E + 1,), 20, dtype=torch.int32, device=DEV)
    offsets[0], offsets[-1] = 0, R
    Y, dX = torch.zeros(R, d_out, dtype=dt, device=DEV), torch.zeros(R, d_in, dtype=dt, device=DEV)
    K.kfac_experts_forward(ctx.h, X, W, offsets, Y)
    K.kfac_experts_input_grad(ctx.h, G, W, offsets, dX)
    eps = 2.0 ** -8 if bf16 else 2.0 ** -24
    for e, rows in ((0, slice(0, 20)), (-1, slice(20, R))):
        for got, a, w in ((Y[rows], X[rows], W[e].double().t()), (dX[rows], G[rows], W[e].double())):
            want, mags = a.double() @ w, a.double().abs() @ w.abs()
            bound = (w.shape[0] + 2) * 2.0 ** -23 * mags + eps * want.abs()
            assert bool(((got.double() - want).abs() <= bound).all())
    del W
    dW = torch.full((E, d_out, d_in), 3.0, device=DEV)
    K.kfac_experts_weight_grad(ctx.h, G, X, offsets, dW)
    for e, rows in ((0, slice(0, 20)), (-1, slice(20, R))):
        g, x = G[rows].double(), X[rows].double()
        assert bool(((dW[e].double() - g.t() @ x).abs() <= (R + 2) * 2.0 ** -23 * (g.abs().t() @ x.abs())).all())
    assert float(dW[1:-1].abs().max()) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_of_more_than_31_bits(ctx, bits):
    """2^31 + 1001 parameters: both ends move as the same elements by themselves, and the state's values at the far end are theirs."""
    n, edge = (1 << 31) + 1001, 1 << 12
    gen = torch.Generator(DEV).manual_seed(7)
    far = (1 << 31) - edge
    ends = ((slice(0, edge), slice(0, edge // 128)), (slice(far, n), slice(far // 128, (n + 127) // 128)))
    p, g = torch.zeros(n, dtype=torch.bfloat16, device=DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    state = dict(m=torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.uint8, device=DEV))
    state["v"] = torch.zeros_like(state["m"])
    if bits == 8:
        state.update({k: torch.zeros((n + 127) // 128, dtype=torch.uint8, device=DEV) for k in ("m_scale", "v_scale")})
    full = dict(param=p, grad=g, **state)
    for s, _ in ends:
        for t in (p, g):
            t[s] = torch.randn(t[s].numel(), generator=gen, device=DEV).to(t.dtype)
    part = lambda s, b: {k: t[b if k.endswith("scale") else s].clone() for k, t in full.items()}
    parts = [part(s, b) for s, b in ends]
    for step in (1, 2):
        K.kfac_adamw_batched(ctx.h, [full], lr=1e-2, step=step)
        K.kfac_adamw_batched(ctx.h, parts, lr=1e-2, step=step)
    for (s, b), short in zip(ends, parts):
        for k, t in full.items():
            assert torch.equal(t[b if k.endswith("scale") else s], short[k]), k
        assert float(short["m"].float().abs().max()) > 0
    assert float(p[edge:edge + 4096].float().abs().max()) == 0
    if bits == 8:
        out = torch.empty(n, dtype=torch.bfloat16, device=DEV)
        K.kfac_adamw_state_values(ctx.h, full["m"], full["m_scale"], out)
        short = torch.empty(parts[1]["m"].numel(), dtype=torch.bfloat16, device=DEV)
        K.kfac_adamw_state_values(ctx.h, parts[1]["m"], parts[1]["m_scale"], short)
        assert torch.equal(out[ends[1][0]], short) and float(short.float().abs().max()) > 0
