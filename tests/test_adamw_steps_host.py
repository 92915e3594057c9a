"""AdamW steps with each tensor's own number, without a GPU: what is refused before a device is touched, and what gets as far as the device."""
import numpy as np
import pytest

from paper_1912_12055_amd import binding as nb

ARG = nb.NNA_ERR_INVALID_ARG
A, M, V, G, S, W = (k << 20 for k in range(1, 7))  # far apart; they stand for pointers, none of which is used
TWO = [(A, G, 300, nb.NNA_F32), (A + 1200, G + 1200, 128, nb.NNA_F32)]


def call(rows=TWO, steps=(1, 1), steps_dev=None, apart=1):
    p, g, n, types = (np.array([r[k] for r in rows], dtype) for k, dtype in enumerate((np.uint64, np.uint64, np.int64, np.int32)))
    steps = None if steps is None else np.array(steps, np.int64)
    return nb.lib().nna_adamw_steps(*(a.ctypes.data for a in (p, g, n, types)), len(rows), M, V, None, None, None, 1 << 20, None if steps is None else steps.ctypes.data, steps_dev, apart,
                                    1e-3, None, 0.9, 0.999, 1e-8, 0.0, -1, None)


@pytest.mark.parametrize("more", [dict(steps=(1, 0)), dict(steps=(-1, 1)), dict(steps=(0, 5), apart=0), dict(steps=None), dict(steps=None, apart=0), dict(apart=2), dict(apart=-1)])
def test_refusals(more):
    assert call(**more) == ARG and "HIP device" not in nb.nna_last_error(), nb.nna_last_error()


@pytest.mark.parametrize("more", [dict(steps=(1, 900)), dict(steps=(3,), apart=0), dict(steps=None, steps_dev=W), dict(steps=None, steps_dev=W, apart=0),
                                  dict(rows=[(A, G, 300, nb.NNA_F32), (S, 0, 5, nb.NNA_F32)], steps=(1, 0)), dict(rows=[], steps=None)])
def test_numbers_of_steps(more):
    """(A tensor without a gradient may have taken no step yet.)"""
    assert call(**more) == ARG and "HIP device" in nb.nna_last_error(), nb.nna_last_error()
