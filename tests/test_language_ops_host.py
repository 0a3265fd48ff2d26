"""CPU-only checks of dropout, embedding and cross entropy: what the entry points refuse before anything is launched, what the binding
refuses, and the tests' own reference against differences, autograd and the generator's published outputs."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import language_reference as R
from tests.test_attention_arguments import OnGpu

OK, INVALID, UNSUPPORTED, WORKSPACE, NULL = 0, 1, 2, 3, 4
A = 1 << 20            # a place for tensors that nothing reads


def test_struct_layout_matches_header():
    # field order and sizes as in the header (LP64)
    assert C.sizeof(B.hbp_rows) == 16 and C.sizeof(B.hbp_dropout_desc) == 8 + 8 * 3
    assert C.sizeof(B.hbp_embedding_desc) == 4 * 4 + 8 * 3 + 32 and C.sizeof(B.hbp_embedding_buffers) == 8 + 8 + 16 * 4 + 8 * 2
    assert C.sizeof(B.hbp_cross_entropy_desc) == 4 * 6 + 8 * 3 and C.sizeof(B.hbp_cross_entropy_buffers) == 8 + 16 * 2 + 8 * 3 + 16 * 2 + 8 * 2


def rows(data=A, stride=1024):
    return B.hbp_rows(data, stride)


def drop_desc(**kw):
    f = dict(struct_size=C.sizeof(B.hbp_dropout_desc), rate=0.25, seed=1, offset=0, counter=None)
    f.update(kw)
    return B.hbp_dropout_desc(*f.values())


def call_dropout(n=0, width=64, dtype=B.BF16, x=None, residual=None, out=None, **kw):
    x, out = x or rows(), out or rows(A << 4)
    return B.lib().hbp_dropout(C.byref(drop_desc(**kw)), dtype, n, width, C.byref(x), None if residual is None else C.byref(residual),
                               C.byref(out), None)


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(struct_size=8), INVALID), (dict(rate=1.0), INVALID), (dict(rate=-0.1), INVALID), (dict(rate=math.nan), INVALID),
    (dict(rate=0.999999), INVALID), (dict(rate=0.99999), OK), (dict(rate=0.0), OK), (dict(counter=A + 4), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(n=-1), INVALID), (dict(width=0), INVALID), (dict(width=-8), INVALID), (dict(width=60), UNSUPPORTED), (dict(width=65544), UNSUPPORTED),
    (dict(n=(1 << 24) + 1), UNSUPPORTED), (dict(n=1 << 24, width=1032), UNSUPPORTED), (dict(n=1, x=rows(0)), NULL), (dict(n=1, out=rows(0)), NULL),
    (dict(n=1, x=rows(A + 2)), UNSUPPORTED), (dict(n=2, x=rows(stride=-8)), INVALID), (dict(n=2, x=rows(stride=65)), UNSUPPORTED),
    (dict(n=2, x=rows(stride=(1 << 22) + 8)), UNSUPPORTED), (dict(n=2, out=rows(stride=56)), INVALID), (dict(n=2, out=rows(stride=0)), INVALID),
    (dict(n=2, x=rows(A, 128), out=rows(A, 64)), INVALID), (dict(n=2, residual=rows(A, 128), out=rows(A, 64)), INVALID),
    (dict(n=2, residual=rows(0)), NULL), (dict(n=2, residual=rows(A + 8)), UNSUPPORTED),
])
def test_dropout_refusals(kw, status):
    assert call_dropout(**kw) == status


def test_missing_descriptors():
    L, r = B.lib(), C.byref(rows())
    assert L.hbp_dropout(None, 1, 0, 64, r, None, r, None) == NULL
    assert L.hbp_dropout(C.byref(drop_desc()), 1, 0, 64, None, None, r, None) == NULL
    assert L.hbp_embedding_workspace_size(None, C.byref(C.c_size_t(0))) == NULL
    assert L.hbp_embedding_workspace_size(C.byref(emb_desc()), None) == NULL
    assert L.hbp_cross_entropy_workspace_size(None, 1, C.byref(C.c_size_t(0))) == NULL
    assert L.hbp_cross_entropy_workspace_size(C.byref(loss_desc()), 1, None) == NULL
    assert L.hbp_embedding_forward(C.byref(emb_desc()), None, None) == NULL
    assert L.hbp_loss_cross_entropy(C.byref(loss_desc()), None, None) == NULL


def emb_desc(**kw):
    f = dict(struct_size=C.sizeof(B.hbp_embedding_desc), dtype=B.BF16, grad_dtype=B.F32, scale=1.0, rows=0, vocab=100, width=64,
             dropout=B.hbp_dropout_desc())
    f.update(kw)
    return B.hbp_embedding_desc(*f.values())


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(struct_size=8), INVALID), (dict(dtype=2), INVALID), (dict(grad_dtype=2), INVALID), (dict(grad_dtype=B.BF16), OK),
    (dict(dtype=B.F32, grad_dtype=B.BF16), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=-2.0), OK),
    (dict(scale=0.0), OK), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(width=0), INVALID), (dict(width=12), UNSUPPORTED),
    (dict(rows=(1 << 24) + 1), UNSUPPORTED), (dict(vocab=(1 << 24) + 1), UNSUPPORTED), (dict(rows=1 << 24, width=1024), OK), (dict(rows=1 << 24, width=1032), UNSUPPORTED),
    (dict(dropout=drop_desc()), OK), (dict(dropout=drop_desc(rate=1.5)), INVALID), (dict(dropout=drop_desc(struct_size=0)), INVALID),
    (dict(dropout=drop_desc(struct_size=0, rate=0.0)), OK), (dict(scale=3e38, dropout=drop_desc(rate=0.9)), INVALID),
])
def test_embedding_descriptor(kw, status):
    n = C.c_size_t(0)
    assert B.lib().hbp_embedding_workspace_size(C.byref(emb_desc(**kw)), C.byref(n)) == status


def emb_bufs(d, **kw):
    n = C.c_size_t(0)
    B.lib().hbp_embedding_workspace_size(C.byref(d), C.byref(n))
    f = dict(struct_size=C.sizeof(B.hbp_embedding_buffers), tokens=A, table=rows(), out=rows(A << 1), dout=rows(A << 2), dtable=rows(A << 3),
             workspace=A << 4, workspace_bytes=n.value)
    f.update(kw)
    return B.hbp_embedding_buffers(*f.values())


@pytest.mark.parametrize("kw,forward,backward", [
    (dict(struct_size=8), INVALID, INVALID), (dict(tokens=None), NULL, NULL), (dict(tokens=A + 2), UNSUPPORTED, UNSUPPORTED),
    (dict(table=rows(0)), NULL, None), (dict(table=rows(stride=-8)), INVALID, None), (dict(out=rows(0)), NULL, None),
    (dict(out=rows(A, 0)), INVALID, None), (dict(dout=rows(0)), None, NULL), (dict(dtable=rows(0)), None, NULL),
    (dict(dtable=rows(A, 0)), None, INVALID), (dict(dtable=rows(A + 4)), None, UNSUPPORTED), (dict(workspace=None), None, WORKSPACE),
    (dict(workspace_bytes=16), None, WORKSPACE), (dict(workspace=A + 8), None, UNSUPPORTED),
])
def test_embedding_refusals(kw, forward, backward):
    d = emb_desc(rows=5)
    if forward is not None:
        assert B.lib().hbp_embedding_forward(C.byref(d), C.byref(emb_bufs(d, **kw)), None) == forward
    if backward is not None:
        assert B.lib().hbp_embedding_backward(C.byref(d), C.byref(emb_bufs(d, **kw)), 0, None) == backward


def test_embedding_accumulate_is_a_truth_value():
    d = emb_desc(rows=5)
    assert B.lib().hbp_embedding_backward(C.byref(d), C.byref(emb_bufs(d)), 2, None) == INVALID


def loss_desc(**kw):
    f = dict(struct_size=C.sizeof(B.hbp_cross_entropy_desc), dtype=B.BF16, grad_dtype=B.F32, mean=1, scale=1.0, factor=1.0, rows=0, vocab=100,
             width=64)
    f.update(kw)
    return B.hbp_cross_entropy_desc(*f.values())


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(struct_size=8), INVALID), (dict(dtype=2), INVALID), (dict(grad_dtype=3), INVALID),
    (dict(dtype=B.F32, grad_dtype=B.BF16), INVALID), (dict(mean=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(factor=math.inf), INVALID), (dict(factor=-1.0), OK), (dict(rows=-1), INVALID),
    (dict(vocab=0), INVALID), (dict(width=0), INVALID), (dict(width=4), UNSUPPORTED), (dict(width=65544), UNSUPPORTED),
    (dict(rows=(1 << 20) + 1), UNSUPPORTED), (dict(vocab=(1 << 24) + 1), UNSUPPORTED),
])
def test_cross_entropy_descriptor(kw, status):
    n = C.c_size_t(0)
    assert B.lib().hbp_cross_entropy_workspace_size(C.byref(loss_desc(**kw)), 1, C.byref(n)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(loss=None), NULL), (dict(targets=None), NULL), (dict(targets=A + 1), UNSUPPORTED),
    (dict(x=rows(0)), NULL), (dict(x=rows(stride=-8)), INVALID), (dict(weight=rows(0)), NULL), (dict(weight=rows(stride=20)), UNSUPPORTED),
    (dict(dx=rows(A + 4)), UNSUPPORTED), (dict(dx=rows(A, 0)), INVALID), (dict(dweight=rows(A, 32)), INVALID), (dict(workspace=None), WORKSPACE),
    (dict(workspace_bytes=64), WORKSPACE), (dict(workspace=A + 8), UNSUPPORTED), (dict(row_loss=A + 2), UNSUPPORTED),
])
def test_cross_entropy_refusals(kw, status):
    d = loss_desc(rows=5)
    n = C.c_size_t(0)
    assert B.lib().hbp_cross_entropy_workspace_size(C.byref(d), 1, C.byref(n)) == OK
    f = dict(struct_size=C.sizeof(B.hbp_cross_entropy_buffers), x=rows(), weight=rows(A << 1), targets=A, loss=A, row_loss=A, dx=rows(A << 2),
             dweight=rows(A << 3), workspace=A << 4, workspace_bytes=n.value)
    f.update(kw)
    assert B.lib().hbp_loss_cross_entropy(C.byref(d), C.byref(B.hbp_cross_entropy_buffers(*f.values())), None) == status


def test_the_loss_alone_needs_less_room():
    n = [C.c_size_t(0), C.c_size_t(0)]
    for g in (0, 1):
        assert B.lib().hbp_cross_entropy_workspace_size(C.byref(loss_desc(rows=1000, vocab=5000)), g, C.byref(n[g])) == OK
    assert 0 < n[0].value < n[1].value


# ---- what the binding refuses -------------------------------------------------------------------------------------
def test_binding_refuses_tensors_that_do_not_fit():
    t, x = OnGpu((6, 16)), OnGpu((5, 16))
    tokens = OnGpu((5,), torch.int32)
    d = loss_desc(dtype=B.F32, rows=5, vocab=6, width=16)
    good = dict(x=x, weight=t, targets=tokens, loss=OnGpu((1,)), row_loss=OnGpu((5,)), dx=OnGpu((5, 16)), dweight=OnGpu((6, 16)),
                workspace=OnGpu((B.cross_entropy_workspace_size(d, True),), torch.uint8))
    B.CrossEntropy(d, **good).buffers()
    for name, bad in (("weight", OnGpu((6, 24))), ("weight", OnGpu((6, 16), torch.bfloat16)), ("targets", OnGpu((5,), torch.int64)),
                      ("targets", OnGpu((4,), torch.int32)), ("loss", None), ("loss", OnGpu((1,), torch.float64)), ("dx", OnGpu((5, 8))),
                      ("dweight", OnGpu((6, 16), torch.bfloat16)), ("row_loss", OnGpu((6,))), ("x", OnGpu((5, 16), device=-1)),
                      ("dx", OnGpu((5, 16), device=1)), ("workspace", OnGpu((64,), torch.uint8, device=-1))):
        with pytest.raises(ValueError, match=name):
            B.CrossEntropy(d, **dict(good, **{name: bad})).buffers()
    e = emb_desc(dtype=B.F32, rows=5, vocab=6, width=16)
    good = dict(tokens=tokens, table=t, out=x, dtable=OnGpu((6, 16)), workspace=OnGpu((1 << 20,), torch.uint8))
    B.Embedding(e, **good).buffers()
    B.Embedding(e, **good).buffers(x)
    for name, bad in (("tokens", OnGpu((5,), torch.int64)), ("out", OnGpu((6, 16))), ("table", OnGpu((6, 16), device=-1))):
        with pytest.raises(ValueError, match=name):
            B.Embedding(e, **dict(good, **{name: bad})).buffers()
    with pytest.raises(ValueError, match="dout"):
        B.Embedding(e, **good).buffers(OnGpu((4, 16)))
    with pytest.raises(ValueError, match="dtable"):
        B.Embedding(e, **dict(good, dtable=None)).buffers(x)
    with pytest.raises(ValueError, match="counter"):
        B.Embedding(e, **good, dropout=B.make_dropout(0.1, 1, counter=OnGpu((1,), torch.int32))).buffers()
    for kw in (dict(seed=-1), dict(seed=1 << 64), dict(seed=0, offset=-1)):
        with pytest.raises(ValueError):
            B.make_dropout(0.1, **kw)


# ---- the tests' own reference -------------------------------------------------------------------------------------
def test_philox_known_answers():
    """The known answers published with the generator (10 rounds; key and counter all zeros, all ones, digits of pi)."""
    ones = 0xFFFFFFFF
    assert R.philox((0, 0), (0, 0, 0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert R.philox((ones, ones), (ones,) * 4) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert R.philox((0xA4093822, 0x299F31D0), (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_reference_mask_is_the_generators():
    seed, offset = 0x123456789ABCDEF0, 0xFEDCBA9876543210
    got = R.kept(3, 16, 0.3, seed, offset)
    for i in range(48):
        w = R.philox((seed & 0xFFFFFFFF, seed >> 32), (i // 8, 0, offset & 0xFFFFFFFF, offset >> 32))[i % 8 // 2]
        assert bool(got[i // 16, i % 16]) == ((w >> (16 * (i % 2)) & 0xFFFF) >= R.threshold(0.3))
    share = R.kept(1000, 1000, 0.3, 5, 1).double().mean().item()
    assert abs(share - (1 - R.threshold(0.3) / 65536)) < 5 * math.sqrt(0.21 / 1e6)       # five standard deviations


@pytest.mark.parametrize("mean", [True, False])
def test_reference_cross_entropy(mean):
    """Values and gradients against torch's own loss and its autograd, and one entry of each against a difference."""
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn((7, 8), generator=g, dtype=torch.float64), torch.randn((11, 8), generator=g, dtype=torch.float64)
    t = torch.tensor([3, -1, 10, 0, 11, 3, 5])
    r = R.cross_entropy(x, w, t, 0.7, mean, 1.5, torch.float64)
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    ignore = torch.where((t >= 0) & (t < 11), t, torch.full_like(t, -100))
    loss = 1.5 * torch.nn.functional.cross_entropy(0.7 * xa @ wa.T, ignore, reduction="mean" if mean else "sum")
    loss.backward()
    assert torch.allclose(r["loss"][0], loss.detach().view(1), rtol=1e-12)
    assert torch.allclose(r["dx"][0], xa.grad, atol=1e-13) and torch.allclose(r["dweight"][0], wa.grad, atol=1e-13)
    h = 1e-5
    for of, i, name in ((x, (2, 3), "dx"), (w, (3, 1), "dweight")):
        value = []
        for d in (h, -h):
            moved = of.clone()
            moved[i] += d
            a = (moved, w) if of is x else (x, moved)
            value.append(R.cross_entropy(*a, t, 0.7, mean, 1.5)["loss"][0].item())
        assert abs((value[0] - value[1]) / (2 * h) - r[name][0][i].item()) < 1e-8


def test_reference_embedding_gradient():
    g = torch.Generator().manual_seed(4)
    table = torch.randn((9, 16), generator=g, dtype=torch.float64).requires_grad_()
    tokens = torch.tensor([2, 2, -1, 8, 9, 0, 2])
    drop = (0.5, 7, 9)
    out, _ = R.embedding(tokens, table.detach(), 3.0, drop)
    ok = (tokens >= 0) & (tokens < 9)
    m = R.multipliers(7, 16, drop, "cpu")
    y = torch.nn.functional.embedding(torch.where(ok, tokens, torch.zeros_like(tokens)), table) * 3.0 * m * ok[:, None]
    assert torch.equal(out, y.detach()) or torch.allclose(out, y.detach(), rtol=1e-15)
    d = torch.randn((7, 16), generator=g, dtype=torch.float64)
    y.backward(d)
    assert torch.allclose(R.embedding_grad(tokens, d, 9, 3.0, drop, torch.float64)[0], table.grad, atol=1e-14)
