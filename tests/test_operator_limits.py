"""What the Python calls for layers of experts and the optimizer step refuse, on the CPU: numbers that the library's types cannot hold."""
import ctypes
import warnings

import pytest
import torch

from paper_2007_00784_amd import kfac as K
from paper_2007_00784_amd.runner import ExpertRunner, device_of

CTX = ctypes.create_string_buffer(4096)


def test_seeds():
    none = (K.kfac_adamw_item * 0)()
    for seed in (-1, 1 << 64):
        with pytest.raises(ValueError, match="seed"):
            K.kfac_adamw_batched(CTX, none, lr=1e-3, seed=seed)


def test_counts_that_no_c_int_holds(monkeypatch):
    """2^32 + 5 rows are not five rows: the library gets a number that it refuses (an address that it could read is 64 here, and no launch follows)."""
    many = (1 << 32) + 5
    assert K.kfac_experts_workspace_bytes(1, many + 300, 70, 1607) == 0 and K.kfac_experts_workspace_bytes(many, 300, 70, 1607) == 0
    assert K.kfac_experts_workspace_bytes(1, 300, 70, (1 << 32) + 1607) == 0 and K.kfac_experts_workspace_bytes(1, 300 - (1 << 32), 70, 1607) == 0 and K.kfac_experts_workspace_bytes(1, 300, 70, 1607) > 0
    monkeypatch.setattr(K, "_on_gpu", lambda *tensors: None)
    monkeypatch.setattr(K, "_ptr", lambda t: 64)
    rows = K._rows
    monkeypatch.setattr(K, "_rows", lambda t, name, d: (128 if name in ("X", "G") else 256, rows(t, name, d)[1]))
    empty = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device="meta")  # noqa: E731
    off = torch.zeros(5, dtype=torch.int32)
    W, X, G = empty(4, 24, 16), empty(many, 16), empty(many, 24)
    calls = [lambda: K.kfac_experts_forward(CTX, X, W, off, G), lambda: K.kfac_experts_input_grad(CTX, G, W, off, X), lambda: K.kfac_experts_weight_grad(CTX, G, X, off, W),
             lambda: K.kfac_update_factors_experts(CTX, X, off, torch.empty(4, 16, 16, device="meta"))]
    for call in calls:
        with pytest.raises(K.KfacError) as e:
            call()
        assert e.value.code == K.KFAC_EINVAL


@pytest.mark.parametrize("bits", [0, 4, 16, 64, "8"])
def test_bits_of_the_optimizer_state(bits):
    """Refused before anything is allocated; they used to mean 32."""
    with pytest.raises(ValueError, match="8 or 32"):
        ExpertRunner(2, 10, 8, 8, state_bits=bits)


def test_the_device_without_a_number(monkeypatch):
    """It is the current one, where torch puts the tensors, not the first."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert device_of("cuda") == torch.device("cuda", 3) and device_of("cuda:1") == torch.device("cuda", 1) and device_of(torch.device("cuda", 2)).index == 2


def test_the_largest_tiles_have_no_parts():
    """However large the workspace is said to be, the plan is that of the size which the query gives."""
    f = K.lib().kfac_experts_plan
    f.argtypes = [ctypes.c_int, ctypes.POINTER(K.kfac_expert_desc), ctypes.c_size_t]
    for shape in ((8, 39084, 24, 3632), (1, 32768, 512, 512), (2, 6000, 75, 133), (16, 32768, 2048, 2048)):
        need = K.kfac_experts_workspace_bytes(*shape, True, K.KFAC_BF16)
        d = ctypes.byref(K.kfac_expert_desc(*shape, 1, K.KFAC_BF16, None))
        for mode in range(4):
            for size in ((1 << 63) - 1, (1 << 64) - 1):
                plan = f(mode, d, size)
                assert plan == f(mode, d, need) and (plan // 100 != 3 or plan % 100 == 1)


def test_a_run_in_8_bits_without_a_seed_is_warned_of_once(monkeypatch):
    """(The item is refused by the library, which is behind the warning.)"""
    def step(told, eight, **kw):
        monkeypatch.setattr(K, "_told", told)
        arr = (K.kfac_adamw_item * 1)(K.kfac_adamw_item(n=-1, m_scale=4096 if eight else None, v_scale=4096 if eight else None))
        with warnings.catch_warnings(record=True) as seen:
            warnings.simplefilter("always")
            with pytest.raises(K.KfacError):
                K.kfac_adamw_batched(CTX, arr, lr=1e-3, **kw)
        return [w.category for w in seen], K._told

    assert step(False, True, step=9) == ([RuntimeWarning], True)
    assert step(True, True, step=10) == ([], True)
    for eight, kw in ((True, dict(step=9, seed=1)), (True, dict(step=8)), (False, dict(step=1000))):
        assert step(False, eight, **kw) == ([], False)
