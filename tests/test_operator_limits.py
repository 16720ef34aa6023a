"""What the Python calls for layers of experts and the optimizer step refuse, on the CPU: numbers that the library's types cannot hold."""
import ctypes

import pytest

from paper_2007_00784_amd import kfac as K

CTX = ctypes.create_string_buffer(4096)


def test_seeds():
    none = (K.kfac_adamw_item * 0)()
    for seed in (-1, 1 << 64):
        with pytest.raises(ValueError, match="seed"):
            K.kfac_adamw_batched(CTX, none, lr=1e-3, seed=seed)
