"""Nothing is written behind the workspaces of the cross entropy and of the embedding's gradient, in any of their forms."""
import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests.test_gpu_language_ops import TYPES, normal, some_tokens

pytestmark = pytest.mark.gpu
BEHIND = 64 << 20           # bytes behind the workspace that are watched


def watched(workspace):
    """A workspace of the same size with bytes behind it, and those."""
    n = workspace.numel()
    whole = torch.full((n + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole[:n], whole[n:]


# logits and sums in one launch; logits in memory; whole tiles and rests; rows filled up; weights copied, one piece and several; shares of both
# gradients; dweight in whole rounds of the compute units; a handful of entries; many pieces of few rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", [(8, 2000, 256), (333, 1009, 72), (100, 30000, 264), (1000, 9300, 128), (600, 40021, 1000), (4090, 9300, 904),
                                           (4100, 22010, 1024), (16384, 33100, 264), (16384, 16, 1024), (5, (2 << 20) + 300, 8), (2049, 1, 8)])
def test_cross_entropy(n, vocab, width, dtype):
    x, w, t = normal((n, width), TYPES[dtype], 1), normal((vocab, width), TYPES[dtype], 2, 0.05), some_tokens(n, vocab, 3)
    for grad in (False, True):
        c = B.make_cross_entropy(x, w, t, grad=grad)
        c.workspace, behind = watched(c.workspace)
        B.hbp_loss_cross_entropy(c)
        assert bool((behind == 0xA5).all()) and bool(torch.isfinite(c.loss).all())


@pytest.mark.parametrize("n,vocab,width", [(1, 1, 8), (4096, 300, 72), (4097, 70000, 264), (70000, 16384, 256), (300000, 77, 64)])
def test_embedding_gradient(n, vocab, width):
    e = B.make_embedding(some_tokens(n, vocab, 1), normal((vocab, width), torch.bfloat16, 2), dropout=B.make_dropout(0.1, 3))
    e.workspace, behind = watched(e.workspace)
    B.hbp_embedding_backward(e, normal((n, width), torch.bfloat16, 4))
    assert bool((behind == 0xA5).all())
