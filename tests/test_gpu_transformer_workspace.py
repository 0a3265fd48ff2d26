"""Deep stacks with shared key/value heads on the GPU: the backward pass takes ever fewer layers at a time, which need more room than all of
them; nothing is written behind the workspace, and the gradients are those of the stack in 64 bits."""
import pytest
import torch

from paper_2501_17086_amd import binding as B, synth
from tests.helpers import TOL, assert_close, to_np
from tests.test_gpu_transformer_positions import BASE, Stack

pytestmark = pytest.mark.gpu
BEHIND = 64 << 20           # bytes behind the workspace that are watched


@pytest.mark.parametrize("sizes,k", [(dict(L=16, N=2048, seq_len=256, d=256, heads=4, kv_heads=2), 4),
                                     (dict(L=34, N=512, seq_len=128, d=512, heads=8, kv_heads=4, rotary=dict(dims=64)), 4)],
                         ids=["8_layers", "17_layers"])
def test_nothing_is_written_behind_the_workspace(sizes, k):
    dtype = "f32"            # (bf16: more layers never share out what fewer do not)
    w = synth.scaled(BASE, dtype=dtype, **sizes)
    inp = synth.make_inputs(w)
    p = B.allocate(w, inp)
    n = p.workspace.numel()
    whole = torch.full((n + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda")
    p.workspace = whole[:n]
    B.hbp_forward(p)
    B.hbp_backward(p, k, gamma=0.2)
    B.hbp_param_grads(p)
    torch.cuda.synchronize()
    assert bool((whole[n:] == 0xA5).all())
    st = Stack(w, inp, torch.arange(w.N) % w.seq_len)
    x = st.run()
    assert_close(to_np(p.x), torch.stack(x).detach().numpy(), TOL[dtype], "x")
    g = st.iterate(k, 0.2)
    assert_close(to_np(p.g), g.detach().numpy(), TOL[dtype], "g")
    for name, want in st.param_grads(g.detach()).items():
        assert_close(to_np(getattr(p, "d" + name)), want.detach().numpy(), TOL[dtype], "d" + name)
