"""CPU-only: what the binding refuses of an attention call's workspace and statistics, with stand-ins for tensors on the GPU."""
import ctypes as C

import pytest
import torch

from paper_2501_17086_amd import binding as B


class OnGpu:
    """Looks like a tensor; nothing reads it."""

    def __init__(self, shape, dtype=torch.float32, device=0, contiguous=True):
        self.shape, self.dtype, self.place, self.contiguous = torch.Size(shape), dtype, device, contiguous
        self.device, self.is_cuda = "cpu" if device < 0 else f"cuda:{device}", device >= 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.place

    def stride(self):
        return tuple(self.shape[i + 1:].numel() for i in range(len(self.shape)))

    def data_ptr(self):
        return 1 << 20


def attention(**kw):
    n, m, H, K, D = 6, 9, 4, 2, 16
    desc = B.hbp_attention_desc(C.sizeof(B.hbp_attention_desc), B.F32, H, K, D, 1, 0.25, 0.0, 1, n, m)
    t = dict(q=OnGpu((n, H, D)), k=OnGpu((m, K, D)), v=OnGpu((m, K, D)), o=OnGpu((n, H, D)), lse=OnGpu((n, H)),
             workspace=OnGpu((B.attention_workspace_size(desc),), torch.uint8))
    t.update(kw)
    return B.Attention(desc, **t)


def test_the_stand_ins_pass_as_they_are():
    b = B.hbp_attention_buffers.from_buffer_copy(attention().buffers())
    assert b.q.data == b.lse == b.workspace == 1 << 20 and b.workspace_bytes == B.attention_workspace_size(attention().desc)
    assert B.hbp_attention_buffers.from_buffer_copy(attention(workspace=None).buffers()).workspace_bytes == 0


@pytest.mark.parametrize("ws", [OnGpu((1 << 16,), torch.uint8, device=-1), OnGpu((1 << 16,), torch.uint8, device=1),
                                OnGpu((1 << 16,), torch.uint8, contiguous=False)], ids=["host", "other_gpu", "strided"])
def test_a_workspace_elsewhere_is_refused(ws):
    with pytest.raises(ValueError, match="workspace"):
        attention(workspace=ws).buffers()


def test_missing_statistics_are_refused():
    with pytest.raises(ValueError, match="lse: .* got none"):
        attention(lse=None).buffers()


@pytest.mark.parametrize("scale,status", [(2.0 ** 127, 0), (2.0 ** 127 * 1.001, 1), (3.0e38, 1)])
def test_a_scale_that_does_not_take_the_exponents_base_is_refused(scale, status):
    """scale log2 e was infinite in fp32, and a score of 0 not a number."""
    n = C.c_size_t(0)
    desc = B.hbp_attention_desc(C.sizeof(B.hbp_attention_desc), B.BF16, 4, 2, 64, 1, scale, 0.0, 1, 8, 8)
    assert B.lib().hbp_attention_workspace_size(C.byref(desc), C.byref(n)) == status
