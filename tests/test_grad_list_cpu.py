"""What the list of gradients for clipping holds on to, on the host: its struct has the buffers' addresses."""
import gc
import weakref

import pytest
import torch

from paper_2110_08450_amd import binding as smfg


class OnDevice(torch.Tensor):
    """A tensor on the host that says it is on the device; nothing here is launched."""
    is_cuda = property(lambda self: True)


def tensor(n, dtype=torch.float32):
    return torch.zeros(n, dtype=dtype).as_subclass(OnDevice)


@pytest.mark.parametrize("change", ["clear", "replace"])
def test_buffers_stay_alive_with_the_list(change):
    """The caller's own lists may be cleared or filled anew."""
    grads, outs, rows = [tensor(40).reshape(4, 10) for _ in range(3)], [None, tensor(40), tensor(40)], [tensor(1, torch.int64), None, tensor(1, torch.int64)]
    kept = [weakref.ref(t) for t in grads + outs + rows if t is not None]
    addresses = [t.data_ptr() for t in grads + outs + rows if t is not None]
    made = smfg.grad_list(grads, outs, rows)
    for given in (grads, outs, rows):
        if change == "clear":
            given.clear()
        else:
            given[:] = [tensor(8) for _ in given]
    gc.collect()
    assert [r().data_ptr() if r() is not None else None for r in kept] == addresses
    assert made.n == 3
