"""Arrays of an AdamW step that share memory, without a GPU: what one workgroup writes while another reads or writes it is refused before a device is touched."""
import numpy as np
import pytest

from paper_1912_12055_amd import binding as nb

F32, BF16 = nb.NNA_F32, nb.NNA_BF16
ARG = nb.NNA_ERR_INVALID_ARG
A, M, V, G, S, W = (k << 20 for k in range(1, 7))  # far apart; they stand for pointers, none of which is used


def call(rows, m=M, v=V, ms=None, vs=None, master=None, step=1, step_dev=None, lr_dev=None):
    """rows: (weights, gradient, values, type)"""
    p, g, n, types = (np.array([r[k] for r in rows], dtype) for k, dtype in enumerate((np.uint64, np.uint64, np.int64, np.int32)))
    return nb.lib().nna_adamw(*(a.ctypes.data for a in (p, g, n, types)), len(rows), m, v, ms, vs, master, 1 << 20, step, step_dev, 1e-3, lr_dev, 0.9, 0.999, 1e-8, 0.0, -1, None)


def call_steps(rows, m=M, v=V, ms=None, vs=None, master=None, steps=None, steps_dev=None, apart=1, lr_dev=None):
    p, g, n, types = (np.array([r[k] for r in rows], dtype) for k, dtype in enumerate((np.uint64, np.uint64, np.int64, np.int32)))
    steps = np.array([1] * len(rows) if steps is None else steps, np.int64)
    return nb.lib().nna_adamw_steps(*(a.ctypes.data for a in (p, g, n, types)), len(rows), m, v, ms, vs, master, 1 << 20, None if steps_dev else steps.ctypes.data, steps_dev, apart, 1e-3,
                                    lr_dev, 0.9, 0.999, 1e-8, 0.0, -1, None)


TWO = [(A, G, 300, F32), (A + 1200, G + 1200, 128, F32)]  # states: 512 values, 2,048 bytes of float32, 512 of codes, 16 of scales
NARROW = [(A, G, 300, BF16), (A + 600, G + 600, 128, BF16)]  # ... and 2,048 bytes of float32 copies
EIGHT = dict(ms=S, vs=S + 4096)


@pytest.mark.parametrize("entry", [call, call_steps])
@pytest.mark.parametrize("rows,more", [
    (TWO, dict(v=M + 512)), (TWO, dict(v=M + 2044)), (TWO, dict(v=M - 2044)), (NARROW, dict(master=M + 4)), (NARROW, dict(master=V - 4)),
    (TWO, dict(v=M + 508, **EIGHT)), (TWO, dict(ms=S, vs=S + 12)), (TWO, dict(ms=M + 100, vs=S)), (TWO, dict(ms=S, vs=V + 508)), (NARROW, dict(master=S - 2044, **EIGHT)),
    # weights over the states
    (TWO, dict(m=A + 1708)), (TWO, dict(v=A - 2044)), (NARROW, dict(master=A + 400)), ([(A, G, 300, F32), (M + 2000, G + 1200, 128, F32)], dict()), (TWO, dict(ms=A + 100, vs=S)),
    # a gradient over another tensor's weights, or its own
    ([(A, G, 300, F32), (S, A + 100, 128, F32)], dict()), ([(A, S + 508, 300, F32), (S, G, 128, F32)], dict()), ([(A, A + 4, 300, F32)], dict()),
    ([(A, A - 2, 300, BF16)], dict()), ([(A, A + 598, 300, BF16), (S, G, 3, F32)], dict()), ([(A, G, 300, BF16), (S, A, 10, BF16), (W, A, 300, BF16)], dict()),
])
def test_shared_memory_is_refused(entry, rows, more):
    assert entry(rows, **more) == ARG and "HIP device" not in nb.nna_last_error(), nb.nna_last_error()


@pytest.mark.parametrize("rows,more", [
    ([(A, M, 300, F32)], dict()), ([(A, M + 1196, 300, F32)], dict()), ([(A, G, 300, F32), (S, V + 1196, 1, F32)], dict()), ([(A, W + 100, 300, BF16)], dict(master=W)),
    ([(A, S + 4, 300, F32)], EIGHT), ([(A, G, 300, F32)], dict(lr_dev=A + 400)), ([(A, G, 300, F32)], dict(steps_dev=A + 1192)), (TWO, dict(steps_dev=V + 2040)),
])
def test_what_the_call_with_each_tensors_step_refuses(rows, more):
    """... and gradients over the states, which nna_adamw leaves to its caller; and numbers in device memory that a workgroup reads while another writes there."""
    assert call_steps(rows, **more) == ARG and "HIP device" not in nb.nna_last_error(), nb.nna_last_error()


@pytest.mark.parametrize("entry", [call, call_steps])
@pytest.mark.parametrize("rows,more", [
    (TWO, dict()), (TWO, dict(v=M + 2048)), (TWO, dict(v=M - 2048)), (TWO, dict(v=M + 512, **EIGHT)), (TWO, dict(ms=S, vs=S + 16)), (TWO, dict(m=A + 1712)),
    (TWO, dict(master=M + 2048)), ([(A, A + 1200, 300, F32), (S, A + 1200, 128, F32)], dict()), ([(A, A + 600, 300, BF16), (S, A - 6, 3, BF16)], dict()),
    # float32 weights have no copies: they may lie where those would be, among 16-bit ones' copies
    ([(W, G, 300, F32), (A, G + 1200, 128, BF16)], dict(master=W)), (TWO, dict(master=A)),
    # states of tensors without a gradient are not written
    ([(A, G, 300, F32), (S, 0, 1000, F32), (W, G, 5, F32)], dict(v=M + 1536)), ([(A, G, 300, F32), (M + 1540, 0, 128, F32), (W, M + 1600, 5, F32)], dict()),
    # a tensor without a gradient is left alone, wherever it is
    ([(A, G, 300, F32), (A + 4, 0, 100, F32), (S, G, 5, F32)], dict()), ([(A, G, 0, F32), (A, A, 0, F32)], dict()),
])
def test_neighbours_are_fine(entry, rows, more):
    assert entry(rows, **more) == ARG and "HIP device" in nb.nna_last_error(), nb.nna_last_error()


@pytest.mark.gpu
def test_tensors_that_share_memory():
    """The same through the binding, of tensors: refused, and nothing is written."""
    import torch

    memory = torch.zeros(4096, device="cuda:0")
    p, g, m, v = memory[:300], memory[512:812], memory[1024:1408], memory[1536:1920]
    master = memory[2048:2432]
    how = dict(params=[p], grads=[g], m=m, v=v, master=master, step=1)
    for bad in (dict(v=memory[1024 + 128 : 1408 + 128]), dict(m=memory[299:683]), dict(grads=[memory[1:301]]), dict(grads=[memory[1400:1700]]),
                dict(params=[p, memory[800:900]], grads=[g, memory[3000:3100]], m=memory[1024:1536], v=memory[1536:2048], master=memory[2048:2560]),
                dict(lr=memory[1030]), dict(step=memory[1536:1538].view(torch.int64))):
        with pytest.raises(nb.NnaError):
            nb.nna_adamw(**{**how, **bad})
    assert not memory.any()
    nb.nna_adamw(**how)
