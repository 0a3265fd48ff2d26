"""A transformer stack allocated with positions of its own, on the GPU."""
import pytest
import torch

from paper_2501_17086_amd import binding as B, synth
from tests.test_gpu_transformer_positions import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", ["shared", "equal_heads"])
def test_positions_given_to_allocate_are_those_of_the_descriptor(case):
    """The same as positions set in the descriptor afterwards; the stack keeps them."""
    w, inp, p = make(case, "bf16")
    pos = ((torch.arange(w.N) * 7) % 53).to(torch.int32)
    keep = pos.cuda()
    p.desc.positions = keep.data_ptr()
    q = B.allocate(w, inp, positions=pos.cuda())
    other = torch.full((w.N,), 999, dtype=torch.int32, device="cuda")          # (would take a freed tensor's place)
    for x in (p, q):
        B.hbp_forward(x)
        B.hbp_backward(x, 2)
        B.hbp_param_grads(x)
    for n in ("x", "qkv", "g", "dWqkv", "dWo"):
        assert torch.equal(getattr(p, n), getattr(q, n)), n
    counted = B.allocate(w, inp)
    B.hbp_forward(counted)
    assert not torch.equal(counted.qkv, q.qkv) and bool((other == 999).all())
    with pytest.raises(ValueError, match="positions"):
        B.allocate(synth.scaled(w, rotary=None), inp, positions=keep)
