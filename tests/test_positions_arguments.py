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


def rotary_status(**kw):
    """Of a call on no rows."""
    r = B.make_rotary(**kw)
    x, y = B.hbp_heads(1 << 20, 1024, 64), B.hbp_heads(1 << 24, 1024, 64)
    return B.lib().hbp_rotary(C.byref(r), B.F32, 0, 4, 64, C.byref(x), C.byref(y), None, 0, 0, 0, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dims=64, base=5e-324), INVALID),                                     # base^(-62/64) passes 2^1023
    (dict(dims=64, base=1e-290), OK),
    (dict(dims=2, base=5e-324), OK),                                           # one pair, which turns by 1 whatever the base
    (dict(dims=64, scaling="linear", factor=1e-300), INVALID), (dict(dims=64, scaling="linear", factor=1e-280), OK),
    (dict(dims=64, scaling="base", factor=1e-300), INVALID),                   # the changed base is 1e-306
    (dict(dims=4, scaling="base", factor=1e-200), INVALID),                    # and here 0
    (dict(dims=64, scaling="by_parts", factor=1e-300, original=64.0), INVALID), (dict(dims=64, scaling="base", factor=1e300), OK),
])
def test_frequencies_that_no_number_holds_are_refused(kw, want):
    """They turned rows into NaN."""
    assert rotary_status(**kw) == want
    n = C.c_size_t(0)
    if kw["dims"] == 64:
        d = B.make_desc(**dict(STACK, d=256), rotary=B.make_rotary(**kw))
        assert status(d) == want


def test_a_stack_has_no_more_turned_heads_than_a_call():
    """Query and key heads are turned together, 65535 at most."""
    wide = dict(STACK, act="gelu", norm="none", L=2, N=32, d=8 * 65535, d_ff=8)
    for heads, want in ((65535, UNSUPPORTED), (32767, OK)):
        sizes = dict(wide, heads=heads, d=8 * heads)
        assert status(B.make_desc(**sizes, rotary=B.make_rotary(8))) == want
        assert status(B.make_desc(**sizes)) == OK
