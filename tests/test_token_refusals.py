"""What the router's choice, the order of tokens, the way back and the gradient norm refuse, on the CPU: every refusal comes before the context is
looked at, so a block of bytes stands for the context and any address for a buffer."""
import contextlib
import ctypes

import pytest
import torch

from paper_2007_00784_amd import kfac as K

CTX = ctypes.create_string_buffer(4096)
A, B, C, D, E, F = (4096 * i for i in range(1, 7))        # addresses that nothing reads
BAD = K.KFAC_EINVAL
NAN, INF = float("nan"), float("inf")


def test_router():
    L = K.lib()
    #            T  E  k  logits dt ldl norm ids weights
    good = dict(T=8, E=16, k=4, logits=A, dt=1, ldl=16, norm=0, ids=B, w=C)

    def forward(ctx=CTX, **kw):
        a = dict(good, **kw)
        return L.kfac_experts_route(ctx, a["T"], a["E"], a["k"], a["logits"], a["dt"], a["ldl"], a["norm"], a["ids"], a["w"])

    def back(ctx=CTX, out=D, ldd=16, **kw):
        a = dict(good, **kw)
        return L.kfac_experts_route_grad(ctx, a["T"], a["E"], a["k"], a["logits"], a["dt"], a["ldl"], a["ids"], a["w"], a["norm"], out, ldd)

    for kw in (dict(T=-1), dict(E=0), dict(E=4097, ldl=5000), dict(k=0), dict(k=17), dict(k=65, E=128, ldl=128), dict(T=1 << 26), dict(logits=None), dict(dt=2), dict(dt=-1), dict(ldl=15),
               dict(ldl=(1 << 20) + 1), dict(norm=2), dict(norm=-1), dict(ids=None), dict(w=None), dict(ids=B + 2), dict(w=C + 1), dict(ctx=None)):
        assert forward(**kw) == BAD, kw
        assert back(**kw) == BAD, kw
    assert forward(ids=A) == BAD and forward(w=A) == BAD and forward(w=B) == BAD
    for kw in (dict(out=None), dict(out=A), dict(out=B), dict(out=C), dict(ldd=15), dict(ldd=(1 << 20) + 1)):
        assert back(**kw) == BAD, kw
    assert forward(T=0, logits=None, ids=None, w=None) == K.KFAC_OK and back(T=0, logits=None, ids=None, w=None, out=None) == K.KFAC_OK


def slots(**kw):
    return ctypes.byref(K.kfac_slot_desc(**dict(dict(tokens=8, topk=2, rows=16, d=64, dtype=1), **kw)))


BAD_SLOTS = [dict(tokens=-1), dict(topk=0), dict(topk=65, rows=1000), dict(tokens=1 << 27, rows=(1 << 28) - 1), dict(rows=-1), dict(rows=1 << 28), dict(d=0), dict(d=65537), dict(dtype=2), dict(dtype=-1)]


@pytest.mark.parametrize("bad", BAD_SLOTS, ids=str)
def test_descriptions_of_slots(bad):
    L = K.lib()
    wide = 1 << 17
    assert L.kfac_experts_dispatch(CTX, slots(**bad), 4, A, B, wide, C, D, E, wide) == BAD
    assert L.kfac_experts_gather(CTX, slots(**bad), A, B, wide, C, wide) == BAD
    assert L.kfac_experts_combine(CTX, slots(**bad), A, B, C, wide, None, 0, D, wide) == BAD
    assert L.kfac_experts_combine_grad(CTX, slots(**bad), A, B, C, wide, D, wide, E, wide, F) == BAD


def test_matrices_of_slots():
    L = K.lib()
    f = L.kfac_experts_dispatch
    #             E  ids X ldx off rows Xs lds
    good = dict(E=4, ids=A, X=B, ldx=64, off=C, rows=D, Xs=E, lds=64)

    def call(desc=None, ctx=CTX, **kw):
        a = dict(good, **kw)
        return f(ctx, desc or slots(), a["E"], a["ids"], a["X"], a["ldx"], a["off"], a["rows"], a["Xs"], a["lds"])

    for kw in (dict(E=0), dict(E=4097), dict(ids=None), dict(X=None), dict(Xs=None), dict(off=None), dict(rows=None), dict(ldx=63), dict(lds=63), dict(ldx=(1 << 20) + 1), dict(lds=(1 << 20) + 1),
               dict(ids=A + 1), dict(off=C + 2), dict(rows=D + 3), dict(rows=A), dict(off=A), dict(off=D), dict(Xs=B), dict(Xs=A), dict(Xs=C), dict(Xs=D), dict(X=C), dict(X=D), dict(ctx=None)):
        assert call(**kw) == BAD, kw
    assert call(slots(rows=15)) == BAD                                     # a row for each slot
    assert f(CTX, None, 4, A, B, 64, C, D, E, 64) == BAD
    f = L.kfac_experts_gather
    for args in ((None, B, 64, C, 64), (A, None, 64, C, 64), (A, B, 64, None, 64), (A, B, 64, B, 64), (A, B, 64, A, 64), (A, B, 63, C, 64), (A, B, 64, C, 63), (A + 2, B, 64, C, 64)):
        assert f(CTX, slots(), *args) == BAD, args
    assert f(None, slots(), A, B, 64, C, 64) == BAD
    assert f(CTX, slots(tokens=0), None, None, 64, None, 64) == K.KFAC_OK and f(CTX, slots(rows=0), A, B, 64, None, 64) == K.KFAC_OK
    f = L.kfac_experts_combine
    for args in ((None, B, C, 64, None, 0, D, 64), (A, B, None, 64, None, 0, D, 64), (A, B, C, 64, None, 0, None, 64), (A, B, C, 64, None, 0, C, 64), (A, B, C, 64, None, 0, A, 64),
                 (A, B, C, 64, None, 0, B, 64), (A, B, C, 63, None, 0, D, 64), (A, B, C, 64, None, 0, D, 63), (A, B, C, 64, E, 63, D, 64), (A, B, C, 64, D, 72, D, 64), (A + 1, B, C, 64, None, 0, D, 64),
                 (A, B + 2, C, 64, None, 0, D, 64)):
        assert f(CTX, slots(), *args) == BAD, args
    assert f(CTX, slots(tokens=0), None, None, None, 64, None, 0, None, 64) == K.KFAC_OK
    f = L.kfac_experts_combine_grad
    good = [A, B, C, 64, D, 64, E, 64, F]
    for i in (0, 1, 2, 4, 6, 8):
        assert f(CTX, slots(), *[None if j == i else a for j, a in enumerate(good)]) == BAD, i
    for i in (3, 5, 7):
        assert f(CTX, slots(), *[63 if j == i else a for j, a in enumerate(good)]) == BAD, i
    for out in (6, 8):
        for i in (0, 1, 2, 4):
            assert f(CTX, slots(), *[good[i] if j == out else a for j, a in enumerate(good)]) == BAD, (out, i)
    for i in (0, 1, 8):
        assert f(CTX, slots(), *[a + 2 if j == i else a for j, a in enumerate(good)]) == BAD, i
    assert f(CTX, slots(), A, B, C, 64, D, 64, E, 64, E) == BAD
    assert f(CTX, slots(tokens=0), *[None if a > 64 else a for a in good]) == K.KFAC_OK


def test_workspace_of_an_order():
    f = K.kfac_experts_dispatch_workspace_bytes
    assert f(-1, 2, 4) == f(8, 0, 4) == f(8, 65, 4) == f(8, 2, 0) == f(8, 2, 4097) == f(1 << 27, 2, 4) == f((1 << 32) + 8, 2, 4) == 0
    assert f(512, 2, 64) == f(2048, 2, 512) == 0                                              # few slots need none
    for T, k, e in ((4097, 1, 64), (1100, 2, 513), (16384, 4, 64), (65536, 8, 128), (65536, 8, 4096), ((1 << 25) - 1, 8, 4096), ((1 << 28) - 1, 1, 1)):
        assert 0 < f(T, k, e) <= 4 << 20 and f(T, k, e) % 256 == 0


def grads(item=None, n=1, clip=True, ctx=CTX, max_norm=1.0, scale=None, norm=C, coef=D):
    it = dict(grad=A, grad_dtype=0, out=B, out_dtype=1, n=10)
    it.update(item or {})
    arr = (K.kfac_grad_item * 1)(K.kfac_grad_item(**it))
    f = K.lib().kfac_clip_grads_batched if clip else K.lib().kfac_grad_norm_batched
    return f(ctx, n, arr, max_norm, scale, norm, coef)


def test_norm_and_clip():
    for clip in (False, True):
        for kw in (dict(item=dict(grad=None)), dict(item=dict(n=-1)), dict(item=dict(grad_dtype=2)), dict(n=-1), dict(ctx=None), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=NAN), dict(norm=None),
                   dict(norm=D), dict(scale=C), dict(scale=D), dict(norm=C + 1), dict(coef=D + 2), dict(scale=E + 1)):
            assert grads(clip=clip, **kw) == BAD, kw
        f = K.lib().kfac_clip_grads_batched if clip else K.lib().kfac_grad_norm_batched
        assert f(CTX, 1, None, 1.0, None, C, D) == BAD
    for kw in (dict(item=dict(out=None)), dict(item=dict(out=A)), dict(item=dict(out_dtype=2)), dict(coef=None)):
        assert grads(**kw) == BAD, kw
    f = K.lib().kfac_grad_norm_workspace_bytes
    assert f(-1, None) == 0 and f(1, None) == 0 and f(0, None) == 0
    assert f(1, (K.kfac_grad_item * 1)(K.kfac_grad_item(n=-1))) == 0 and f(1, (K.kfac_grad_item * 1)(K.kfac_grad_item(n=5, grad_dtype=3))) == 0
    assert 0 < f(1, (K.kfac_grad_item * 1)(K.kfac_grad_item(n=5))) < f(1, (K.kfac_grad_item * 1)(K.kfac_grad_item(n=1 << 30))) == 8192


@contextlib.contextmanager
def refused(match=None):
    """Refused, and for what is wrong with the case: that these tensors are not on a GPU is looked at behind everything else."""
    with pytest.raises(ValueError, match=match) as e:
        yield
    assert "GPU" not in str(e.value)


def test_tensors_that_do_not_fit():
    i32, bf = torch.int32, torch.bfloat16
    logits, ids, w = torch.zeros(6, 16), torch.zeros(6, 2, dtype=i32), torch.zeros(6, 2)
    for args in ((logits[:5], ids, w), (logits, ids.long(), w), (logits, ids, w.double()), (logits, ids, w[:, :1]), (logits, ids[:, 0], w), (logits.half(), ids, w), (logits[0], ids, w),
                 (logits, torch.zeros(2, 6, dtype=i32).t(), w), (logits, ids, torch.zeros(2, 6).t()), (torch.zeros(16, 6).t(), ids, w), (logits[:1].expand(6, 16), ids, w)):
        with refused():
            K.kfac_experts_route(CTX, *args)
        with refused():
            K.kfac_experts_route_grad(CTX, *args, torch.zeros(args[0].shape, dtype=args[0].dtype))
    for out in (logits[:5], logits.to(bf), logits[:, :15], logits[0], torch.zeros(16, 6).t()):
        with refused():
            K.kfac_experts_route_grad(CTX, logits, ids, w, out)
    X, Xs, off = torch.zeros(6, 32), torch.zeros(12, 32), torch.zeros(5, dtype=i32)
    for args in ((ids.long(), X, off, ids, Xs), (ids, X[:5], off, ids, Xs), (ids, X, off.long(), ids, Xs), (ids, X, off[:1], ids, Xs), (ids, X, off, ids.long(), Xs), (ids, X, off, ids[:5], Xs),
                 (ids, X, off, ids, Xs[:11]), (ids, X, off, ids, Xs[:, :31]), (ids, X, off, ids, Xs.to(bf)), (ids, None, off, ids, Xs), (ids, X, off, ids, None), (ids, X, off[::2], ids, Xs),
                 (ids, X.double(), off, ids, Xs.double()), (ids, X[0], off, ids, Xs)):
        with refused():
            K.kfac_experts_dispatch(CTX, *args)
    for args in ((ids.long(), X, Xs), (ids, X[:5], Xs), (ids, X, Xs.to(bf)), (ids, X, Xs[:, :31])):
        with refused():
            K.kfac_experts_gather(CTX, *args)
    for args, add in (((Xs, ids.long(), w, X), None), ((Xs, ids, w[:, :1], X), None), ((Xs, ids, w.to(bf), X), None), ((Xs, ids, w, X[:5]), None), ((Xs, ids, w, X[:, :31]), None),
                      ((Xs.to(bf), ids, w, X), None), ((Xs, ids, w, X), X[:5]), ((Xs, ids, w, X), X.to(bf)), ((Xs, ids, w, X), X[:, :31]), ((Xs, ids, w, X[0]), None)):
        with refused():
            K.kfac_experts_combine(CTX, *args, add=add)
    for args in ((X, Xs, ids.long(), w, Xs, w), (X, Xs, ids, w[:5], Xs, w), (X, Xs, ids, w, Xs, w[:, :1]), (X[:5], Xs, ids, w, Xs, w), (X, Xs[:11], ids, w, Xs, w), (X, Xs.to(bf), ids, w, Xs, w),
                 (X, Xs, ids, w, Xs.to(bf), w), (X, Xs[:, :31], ids, w, Xs, w), (X, Xs, ids, w, Xs[:, :31], w)):
        with refused():
            K.kfac_experts_combine_grad(CTX, *args)
    for call in (lambda: K.kfac_experts_route(CTX, logits, ids, w), lambda: K.kfac_experts_route_grad(CTX, logits, ids, w, logits.clone()), lambda: K.kfac_experts_dispatch(CTX, ids, X, off, ids.clone(), Xs),
                 lambda: K.kfac_experts_dispatch(CTX, ids, None, off, ids.clone(), None), lambda: K.kfac_experts_gather(CTX, ids, X, Xs), lambda: K.kfac_experts_combine(CTX, Xs, ids, w, X),
                 lambda: K.kfac_experts_combine(CTX, Xs, ids, None, X, add=X), lambda: K.kfac_experts_combine_grad(CTX, X, Xs, ids, w, Xs.clone(), w.clone()),
                 lambda: K.grad_items([X]), lambda: K.grad_items([X], [Xs[:6]]), lambda: K.kfac_grad_norm_batched(CTX, (K.kfac_grad_item * 0)(), torch.zeros(1))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_lists_of_gradients(monkeypatch):
    monkeypatch.setattr(K, "_on_gpu", lambda *tensors: None)
    a, b, c = torch.zeros(10), torch.zeros(20), torch.zeros(10)
    bf = torch.zeros(10, dtype=torch.bfloat16)
    assert len(K.grad_items([a, b])) == len(K.grad_items([a, b], [a, b])) == len(K.grad_items([a, b], [bf, b])) == 2
    assert len(K.grad_items([a, a])) == 2 and len(K.grad_items([a, a], [bf, c])) == 2            # (only read)
    assert len(K.grad_items([a[:0], a], [a[:0], a])) == 2                                        # (nothing in it)
    for g, o in (([a, b], [a]), ([a], [b]), ([a.half()], None), ([a], [a.half()]), ([torch.zeros(20)[::2]], None), ([a], [torch.zeros(20)[::2]])):
        with refused():
            K.grad_items(g, o)
    for g, o in (([a, c], [bf, bf]), ([a, a], [a, a])):
        with refused("twice"):
            K.grad_items(g, o)
    for g, o in (([a, c], [c, a]), ([a, c], [c, bf]), ([a, a], [a, c])):
        with refused("another"):
            K.grad_items(g, o)
    with refused("in place"):
        K.grad_items([a], [a.view(torch.bfloat16)[:10]])
    none = (K.kfac_grad_item * 0)()
    for kw in (dict(norm=torch.zeros(2)), dict(norm=torch.zeros(1).double()), dict(norm=a[:1], coef=torch.zeros(2)), dict(norm=a[:1], grad_scale=bf[:1])):
        with refused():
            K.kfac_grad_norm_batched(CTX, none, **kw)


def test_counts_that_no_c_int_holds(monkeypatch):
    """2^32 + 6 tokens are not six tokens: the library gets a number that it refuses."""
    many = (1 << 32) + 6
    monkeypatch.setattr(K, "_on_gpu", lambda *tensors: None)
    monkeypatch.setattr(K, "_slots", lambda t, name, shape=None, ints=True: (64, t.shape))
    matrix = K._matrix
    monkeypatch.setattr(K, "_matrix", lambda t, name, *a: (128 if name in ("X", "Ys", "logits") else 256,) + matrix(t, name, *a)[1:])
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")  # noqa: E731
    ids, w, X, Xs = empty(many, 2), empty(many, 2), empty(many, 8), empty(2 * many, 8)
    off = torch.zeros(5, dtype=torch.int32)
    for call in (lambda: K.kfac_experts_route(CTX, X, ids, w), lambda: K.kfac_experts_route_grad(CTX, X, ids, w, empty(many, 8)), lambda: K.kfac_experts_dispatch(CTX, ids, X, off, ids, Xs),
                 lambda: K.kfac_experts_gather(CTX, ids, X, Xs), lambda: K.kfac_experts_combine(CTX, Xs, ids, w, X), lambda: K.kfac_experts_combine_grad(CTX, X, Xs, ids, w, Xs, w)):
        with pytest.raises(K.KfacError) as e:
            call()
        assert e.value.code == BAD
