"""What the calls for layers of experts and the optimizer step refuse, on the CPU: every refusal comes before the context is looked at, let
alone a launch, so a block of bytes stands for the context and any address for a buffer."""
import contextlib
import ctypes

import pytest
import torch

from paper_2007_00784_amd import kfac as K

CTX = ctypes.create_string_buffer(4096)
A, B, C, D = 4096, 8192, 12288, 16384        # addresses that nothing reads


def desc(**kw):
    d = dict(experts=4, rows=100, d_in=64, d_out=32, append_ones=0, dtype=K.KFAC_BF16, offsets=D)
    d.update(kw)
    return ctypes.byref(K.kfac_expert_desc(**d))


BAD_DESCS = [dict(experts=0), dict(experts=4097), dict(rows=-1), dict(rows=1 << 28), dict(d_in=0), dict(d_out=0), dict(d_in=65537), dict(d_out=65537),
             dict(append_ones=2), dict(append_ones=-1), dict(dtype=2), dict(offsets=None), dict(offsets=D + 2)]


@pytest.mark.parametrize("bad", BAD_DESCS, ids=str)
def test_descriptions_of_a_layer(bad):
    L = K.lib()
    wide = 1 << 17
    assert L.kfac_experts_forward(CTX, desc(**bad), A, wide, B, C, wide) == K.KFAC_EINVAL
    assert L.kfac_experts_input_grad(CTX, desc(**bad), A, wide, B, C, wide) == K.KFAC_EINVAL
    assert L.kfac_experts_weight_grad(CTX, desc(**bad), A, wide, B, wide, 0, C, K.KFAC_F32) == K.KFAC_EINVAL
    if "d_out" not in bad:
        d = dict(experts=4, rows=100, offsets=D, dtype=K.KFAC_BF16, d_in=64, append_ones=0)
        d.update(bad)
        assert L.kfac_update_factors_experts(CTX, d["experts"], d["rows"], d["offsets"], A, d["dtype"], wide, d["d_in"], d["append_ones"], 1, 1.0, 0.5, C) == K.KFAC_EINVAL


def test_matrices_of_products():
    L = K.lib()
    bad = K.KFAC_EINVAL
    for f in (L.kfac_experts_forward, L.kfac_experts_input_grad):
        assert f(None, desc(), A, 64, B, C, 64) == bad
        assert f(CTX, None, A, 64, B, C, 64) == bad
        assert f(CTX, desc(), None, 64, B, C, 64) == bad
        assert f(CTX, desc(), A, 64, None, C, 64) == bad
        assert f(CTX, desc(), A, 64, B, None, 64) == bad
        assert f(CTX, desc(), A, 64, B, A, 64) == bad          # output on an input
        assert f(CTX, desc(), A, 64, B, B, 64) == bad
        assert f(CTX, desc(), A, 31, B, C, 64) == bad          # pitch below the row
        assert f(CTX, desc(), A, 64, B, C, 31) == bad
        assert f(CTX, desc(), A, (1 << 20) + 1, B, C, 64) == bad
        assert f(CTX, desc(), A, 64, B, C, (1 << 20) + 1) == bad
        assert f(CTX, desc(rows=0), None, 64, B, None, 64) == K.KFAC_OK
    f = L.kfac_experts_weight_grad
    for args in ((None, 64, B, 64, 0, C, 0), (A, 64, None, 64, 0, C, 0), (A, 64, B, 64, 0, None, 0), (A, 64, B, 64, 2, C, 0), (A, 64, B, 64, 0, C, 2),
                 (A, 64, B, 64, 0, A, 0), (A, 64, B, 64, 0, B, 0), (A, 31, B, 64, 0, C, 0), (A, 64, B, 63, 0, C, 0), (A, 64, B, (1 << 20) + 1, 0, C, 0)):
        assert f(CTX, desc(), *args) == bad, args
    f = L.kfac_update_factors_experts
    nan, inf = float("nan"), float("inf")
    #           X  dt ldx d   1s mean scale decay F
    for args in ((None, 1, 64, 64, 0, 1, 1.0, 0.5, C), (A, 1, 64, 64, 0, 1, 1.0, 0.5, None), (A, 1, 64, 64, 0, 1, 1.0, 0.5, A), (A, 1, 63, 64, 0, 1, 1.0, 0.5, C),
                 (A, 1, 9000, 8193, 0, 1, 1.0, 0.5, C), (A, 1, 9000, 8192, 1, 1, 1.0, 0.5, C), (A, 1, 64, 64, 0, 2, 1.0, 0.5, C), (A, 1, 64, 64, 0, 1, nan, 0.5, C),
                 (A, 1, 64, 64, 0, 1, inf, 0.5, C), (A, 1, 64, 64, 0, 1, 1.0, -0.1, C), (A, 1, 64, 64, 0, 1, 1.0, 1.1, C), (A, 1, 64, 64, 0, 1, 1.0, nan, C)):
        assert f(CTX, 4, 100, D, *args) == bad, args
    assert f(None, 4, 100, D, A, 1, 64, 64, 0, 1, 1.0, 0.5, C) == bad


def adamw(item=None, opts=None, n=1, ctx=CTX):
    it = dict(param=A, param_dtype=0, grad=B, grad_dtype=0, m=C, v=D, m_scale=None, v_scale=None, copy=None, n=10)
    it.update(item or {})
    o = dict(beta1=0.9, beta2=0.999, lr=1e-3, eps=1e-8, weight_decay=0.0, step=1)
    o.update(opts or {})
    return K.lib().kfac_adamw_batched(ctx, n, (K.kfac_adamw_item * 1)(K.kfac_adamw_item(**it)), ctypes.byref(K.kfac_adamw_opts(**o)))


def test_optimizer_step():
    bad = K.KFAC_EINVAL
    for item in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(param_dtype=2), dict(grad_dtype=-1), dict(m_scale=A + 1), dict(v_scale=A + 1),
                 dict(m_scale=A + 1, v_scale=A + 1), dict(v=C), dict(grad=A), dict(m=A), dict(v=A), dict(copy=A), dict(copy=B), dict(copy=C), dict(copy=D), dict(grad=C), dict(grad=D)):
        assert adamw(item) == bad, item
    nan, inf = float("nan"), float("inf")
    for opts in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1e-8), dict(eps=nan), dict(eps=inf), dict(weight_decay=-0.1),
                 dict(weight_decay=nan), dict(weight_decay=inf), dict(lr=nan), dict(lr=inf), dict(step=0), dict(step=-3)):
        assert adamw(opts=opts) == bad, opts
    assert adamw(n=-1) == bad and adamw(ctx=None) == bad
    L = K.lib()
    assert L.kfac_adamw_batched(CTX, 1, None, ctypes.byref(K.kfac_adamw_opts(beta1=0.9, beta2=0.9, step=1))) == bad
    assert L.kfac_adamw_batched(CTX, 0, None, None) == bad
    f = L.kfac_adamw_state_values
    assert f(CTX, A, B, 10, C, 2) == bad and f(CTX, A, B, -1, C, 0) == bad and f(None, A, B, 10, C, 0) == bad
    assert f(CTX, None, B, 10, C, 0) == bad and f(CTX, A, None, 10, C, 0) == bad and f(CTX, A, B, 10, None, 0) == bad
    assert f(CTX, A, B, 10, A, 0) == bad and f(CTX, A, B, 10, B, 0) == bad
    assert f(CTX, None, None, 0, None, 0) == K.KFAC_OK


@contextlib.contextmanager
def refused():
    """Refused, and for what is wrong with the case: that these tensors are not on a GPU is looked at behind everything else."""
    with pytest.raises(ValueError) as e:
        yield
    assert "GPU" not in str(e.value)


def test_tensors_that_do_not_fit():
    off = torch.zeros(5, dtype=torch.int32)
    X, W, Y = torch.zeros(10, 16), torch.zeros(4, 24, 16), torch.zeros(10, 24)
    bf = torch.bfloat16
    for args in ((X, W, off[:4], Y), (X, W, off.long(), Y), (X, W, off, Y[:9]), (X, W, off, Y[:, :23]), (X[:, :15], W, off, Y), (X, W.to(bf), off, Y),
                 (X, W, off, Y.to(bf)), (X.double(), W.double(), off, Y.double()), (torch.zeros(16, 10).t(), W, off, Y), (X[:1].expand(10, 16), W, off, Y),
                 (X, W.transpose(1, 2).contiguous().transpose(1, 2), off, Y)):
        with refused():
            K.kfac_experts_forward(CTX, *args)
    for args in ((Y, W, off, X[:, :15]), (Y[:9], W, off, X), (Y[:, :20], W, off, X), (Y.to(bf), W, off, X)):
        with refused():
            K.kfac_experts_input_grad(CTX, *args)
    for args in ((Y, X, off, W[:, :, :15]), (Y[:9], X, off, W), (Y, X.to(bf), off, W), (Y, X, off, W.half())):
        with refused():
            K.kfac_experts_weight_grad(CTX, *args)
    F = torch.zeros(4, 16, 16)
    for args, kw in (((X, off, F), dict(append_ones=True)), ((X, off, F.to(bf)), {}), ((X, off[:3], F), {}), ((X, off, F[:, :15, :15]), {})):
        with refused():
            K.kfac_update_factors_experts(CTX, *args, **kw)
    p, u = torch.zeros(300), torch.zeros(300, dtype=torch.uint8)
    s = torch.zeros(3, dtype=torch.uint8)
    good = dict(param=p, grad=p, m=p, v=p)
    eight = dict(param=p, grad=p, m=u, v=u, m_scale=s, v_scale=s)
    for it in (dict(good, grad=p[:299]), dict(good, m=u), dict(good, m_scale=s), dict(eight, m=p), dict(eight, m_scale=s[:2]), dict(eight, v_scale=p[:3]), dict(good, copy=p),
               dict(good, copy=torch.zeros(299, dtype=bf)), dict(good, param=p.half()), dict(good, grad=torch.zeros(600)[::2])):
        with refused():
            K.adamw_items([it])
    for kw in (dict(lr=torch.zeros(2)), dict(lr=1e-3, step=torch.zeros(1)), dict(lr=1e-3, grad_scale=torch.zeros(1, dtype=bf))):
        with refused():
            K.kfac_adamw_batched(CTX, (K.kfac_adamw_item * 1)(), **kw)
    for args in ((u, s[:2], p), (u, s, p[:299]), (p, s, p), (u, s, p.half())):
        with refused():
            K.kfac_adamw_state_values(CTX, *args)
    for call in (lambda: K.kfac_experts_forward(CTX, X, W, off, Y), lambda: K.kfac_experts_input_grad(CTX, Y, W, off, X), lambda: K.kfac_experts_weight_grad(CTX, Y, X, off, W),
                 lambda: K.kfac_update_factors_experts(CTX, X, off, F), lambda: K.adamw_items([good]), lambda: K.adamw_items([eight]), lambda: K.kfac_adamw_state_values(CTX, u, s, p)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_codes_of_another_format():
    """One byte an element is not enough: only e4m3 codes are what the state holds."""
    p, s = torch.zeros(300), torch.zeros(3, dtype=torch.uint8)
    for dt in (torch.float8_e5m2, torch.float8_e4m3fnuz, torch.int8, torch.bool):
        u = torch.zeros(300).to(dt)
        for pair in ((u, torch.zeros(300, dtype=torch.uint8)), (torch.zeros(300, dtype=torch.uint8), u)):
            with refused():
                K.adamw_items([dict(param=p, grad=p, m=pair[0], v=pair[1], m_scale=s, v_scale=s)])
        with refused():
            K.kfac_adamw_state_values(CTX, u, s, p)


def test_buffers_that_occur_twice(monkeypatch):
    monkeypatch.setattr(K, "_on_gpu", lambda *tensors: None)

    def item(eight=False, n=300):
        new = (lambda: torch.zeros(n, dtype=torch.uint8)) if eight else (lambda: torch.zeros(n))
        it = dict(param=torch.zeros(n), grad=torch.zeros(n), m=new(), v=new(), copy=torch.zeros(n, dtype=torch.bfloat16))
        return dict(it, m_scale=torch.zeros(-(-n // 128), dtype=torch.uint8), v_scale=torch.zeros(-(-n // 128), dtype=torch.uint8)) if eight else it

    for eight in (False, True):
        a, b = item(eight), item(eight)
        assert len(K.adamw_items([a, b, item(eight, 0), item(eight, 0)])) == 4
        assert len(K.adamw_items([a, dict(b, grad=a["grad"])])) == 2       # (a gradient is only read)
        for key in a:
            if key != "grad":
                with pytest.raises(ValueError, match="twice"):
                    K.adamw_items([a, dict(b, **{key: a[key]})])
        with pytest.raises(ValueError, match="twice"):
            K.adamw_items([dict(a, m=a["v"])])


def test_the_pitch_of_a_single_row():
    """One row has no pitch, whatever the matrix was that it is taken from."""
    assert K._rows(torch.empty(1 << 21).as_strided((1, 8), (1 << 21, 1)), "X", 8)[1] == 8
    assert K._rows(torch.empty(16).as_strided((1, 8), (0, 1)), "X", 8)[1] == 8
    assert K._rows(torch.empty(32).as_strided((2, 8), (16, 1)), "X", 8)[1] == 16


def test_workspace_of_experts():
    """What is asked for suffices for the plan, less of it means fewer parts, and an invalid description asks for nothing."""
    f = K.lib().kfac_experts_plan
    f.argtypes = [ctypes.c_int, ctypes.POINTER(K.kfac_expert_desc), ctypes.c_size_t]
    for dtype in (K.KFAC_F32, K.KFAC_BF16):
        for shape in ((1, 32768, 512, 512), (2, 6000, 75, 133), (1, 300, 70, 1607), (64, 4096, 2048, 1000), (3, 1, 8, 8), (1, (1 << 28) - 1, 64, 64), (4096, 0, 65536, 65536)):
            for ones in (0, 1):
                need = K.kfac_experts_workspace_bytes(*shape, ones, dtype)
                assert need % 256 == 0 and need < 1 << 31
                for mode in range(4):
                    d = ctypes.byref(K.kfac_expert_desc(*shape, ones, dtype, None))
                    full, some, none = f(mode, d, 1 << 60), f(mode, d, need // 3), f(mode, d, 0)
                    assert f(mode, d, need) == full
                    assert none % 100 == 1 and (some // 100 != full // 100 or some % 100 <= full % 100)
    assert K.kfac_experts_workspace_bytes(0, 100, 64, 64) == 0 and K.kfac_experts_workspace_bytes(1, -1, 64, 64) == 0


TILE_OF = ((16, 32, 256), (32, 64, 256), (32, 32, 256), (256, 256, 512), (128, 128, 256), (128, 128, 256), (32, 64, 256))      # rows, columns, threads of an engine


@pytest.mark.parametrize("dtype", [K.KFAC_F32, K.KFAC_BF16])
@pytest.mark.parametrize("mode", [0, 1])
def test_long_layers_fit_a_launch(dtype, mode):
    """Whatever fits the memory (288 GB) runs: an engine is taken only if its workgroups are fewer than a launch can have (2^32 threads)."""
    f = K.lib().kfac_experts_plan
    f.argtypes = [ctypes.c_int, ctypes.POINTER(K.kfac_expert_desc), ctypes.c_size_t]
    taken = set()
    for rows in (1 << 20, 1 << 24, (1 << 28) - 1):
        for side in (4, 8, 16, 64, 128, 256, 1000, 4096):
            for other in (4, 8, 64, 1000, 4096):
                for experts in (1, 64, 4096):
                    if (2 if dtype else 4) * (rows * (side + other) + experts * side * other) > 288e9:
                        continue
                    engine = f(mode, ctypes.byref(K.kfac_expert_desc(experts, rows, side, other, 0, dtype, None)), 0) // 100
                    r, c, threads = TILE_OF[engine]
                    cols = other if mode == 0 else side
                    tiles = (rows // r + min(experts, rows)) * -(-cols // c)
                    assert -(-tiles // 8) * 8 * threads < 1 << 32, (rows, side, other, experts, engine)
                    taken.add(engine)
    assert len(taken) > 1
