"""CPU-only: what is refused of the positions that a transformer stack is given, and of rotary descriptors."""
import ctypes as C

import pytest
import torch

from paper_2501_17086_amd import binding as B

OK, INVALID, UNSUPPORTED = 0, 1, 2
STACK = dict(kind="transformer", dtype="bf16", act="gelu", norm="rms", L=4, N=64, d=128, d_ff=256, heads=4, seq_len=32)


def status(desc):
    n = C.c_size_t(0)
    return B.lib().hbp_workspace_size(C.byref(desc), C.byref(n))


class OnGpu:
    """Looks like a tensor on the GPU; nothing reads it."""

    def __init__(self, shape, dtype=torch.int32, contiguous=True):
        self.shape, self.dtype, self.contiguous, self.device, self.is_cuda = torch.Size(shape), dtype, contiguous, "cuda:0", True

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return 0

    def stride(self):
        return (1,) * len(self.shape)

    def data_ptr(self):
        return 1 << 20


def test_positions_of_a_stack_are_refused_where_nothing_turns():
    given = OnGpu((64,))
    for kw in (dict(), dict(kv_heads=2), dict(kv_heads=4)):
        with pytest.raises(ValueError, match="positions"):
            B.make_desc(**STACK, positions=given, **kw)
    d = B.make_desc(**STACK, kv_heads=2)
    assert status(d) == OK
    d.positions = 1 << 20
    assert status(d) == INVALID
    d = B.make_desc(**STACK, rotary=B.make_rotary(32), positions=given)
    assert d.positions == 1 << 20 and status(d) == OK


@pytest.mark.parametrize("bad", [torch.zeros(64, dtype=torch.int32), OnGpu((64,), torch.int64), OnGpu((63,)), OnGpu((64, 1)),
                                 OnGpu((64,), contiguous=False)], ids=["host", "int64", "short", "two_dimensions", "strided"])
def test_positions_of_a_stack_are_one_int32_for_every_token(bad):
    with pytest.raises(ValueError, match="positions"):
        B.make_desc(**STACK, rotary=B.make_rotary(32), positions=bad)
