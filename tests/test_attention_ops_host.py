"""CPU-only checks of the rotary and attention entry points: what they refuse before anything is launched, and the tests'
own reference against plain differences and torch's autograd."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import attention_reference as R

OK, INVALID, UNSUPPORTED, WORKSPACE, NULL = 0, 1, 2, 3, 4
A = 1 << 20            # a place for tensors that nothing reads


def heads(data=A, row=1024, head=64):
    return B.hbp_heads(data, row, head)


def call_rotary(rot=None, dtype=B.BF16, rows=0, n=4, dh=64, x=None, out=None, positions=None, first=0, period=0, inverse=0, **kw):
    rot = B.make_rotary(**dict(dict(dims=64), **kw)) if rot is None else rot
    x = heads() if x is None else x
    out = heads(A << 4) if out is None else out
    return B.lib().hbp_rotary(C.byref(rot), dtype, rows, n, dh, C.byref(x), C.byref(out), positions, first, period, inverse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(dims=0), INVALID), (dict(dims=7), INVALID), (dict(dims=66), INVALID), (dict(dims=-2), INVALID),
    (dict(base=0.0), INVALID), (dict(base=math.inf), INVALID), (dict(base=math.nan), INVALID), (dict(magnitude=math.nan), INVALID),
    (dict(scaling="linear", factor=0.0), INVALID), (dict(scaling="linear", factor=math.inf), INVALID),
    (dict(scaling="base", factor=2.0, dims=2), INVALID), (dict(scaling="base", factor=2.0, dims=4), OK),
    (dict(scaling="by_parts", factor=2.0), INVALID), (dict(scaling="by_parts", factor=2.0, original=64, low=4, high=4), INVALID),
    (dict(scaling="by_parts", factor=2.0, original=64), OK),
    (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(n=0), INVALID), (dict(period=-1), INVALID), (dict(inverse=2), INVALID),
    (dict(dh=60, dims=16), UNSUPPORTED), (dict(dh=264), UNSUPPORTED), (dict(dh=256), OK), (dict(rows=(1 << 24) + 1), UNSUPPORTED),
    (dict(rows=1, x=heads(0)), NULL), (dict(rows=1, x=heads(A + 2)), UNSUPPORTED), (dict(rows=2, x=heads(row=-8)), INVALID),
    (dict(rows=1, x=heads(head=65)), UNSUPPORTED), (dict(rows=2, x=heads(row=1 << 24)), UNSUPPORTED),
    (dict(rows=1, out=heads(head=0)), INVALID), (dict(rows=3, out=heads(row=128)), INVALID),
    (dict(rows=2, x=heads(A, 512, 64), out=heads(A, 256, 64)), INVALID),
])
def test_rotary_refusals(kw, status):
    assert call_rotary(**kw) == status


def test_rotary_refusals_of_the_descriptor_itself():
    r = B.make_rotary(64)
    for field, value in (("struct_size", 8), ("layout", 2), ("scaling", 4), ("reserved", 1.0)):
        bad = B.hbp_rotary_desc.from_buffer_copy(r)
        setattr(bad, field, value)
        assert call_rotary(bad) == INVALID
    assert B.lib().hbp_rotary(None, 1, 0, 1, 64, C.byref(heads()), C.byref(heads()), None, 0, 0, 0, None) == NULL
    assert B.lib().hbp_rotary(C.byref(r), 1, 0, 1, 64, None, C.byref(heads()), None, 0, 0, 0, None) == NULL


def desc(**kw):
    f = dict(struct_size=C.sizeof(B.hbp_attention_desc), dtype=B.BF16, heads=8, kv_heads=2, dh=64, causal=1, scale=0.125, reserved=0.0,
             seqs=2, q_rows=64, k_rows=64)
    f.update(kw)
    return B.hbp_attention_desc(*f.values())


@pytest.mark.parametrize("kw,status", [
    (dict(), OK), (dict(struct_size=4), INVALID), (dict(dtype=2), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(kv_heads=3), INVALID), (dict(kv_heads=16), INVALID), (dict(dh=0), INVALID), (dict(dh=60), UNSUPPORTED),
    (dict(dh=136), UNSUPPORTED), (dict(causal=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(reserved=1.0), INVALID), (dict(seqs=0), INVALID),
    (dict(q_rows=-1), INVALID), (dict(k_rows=-1), INVALID), (dict(q_rows=0, k_rows=0), OK), (dict(q_rows=(1 << 24) + 1), UNSUPPORTED),
    (dict(q_rows=1 << 24, heads=128), UNSUPPORTED),
])
def test_attention_descriptor(kw, status):
    n = C.c_size_t(0)
    assert B.lib().hbp_attention_workspace_size(C.byref(desc(**kw)), C.byref(n)) == status


def buffers(d, **kw):
    n = C.c_size_t(0)
    B.lib().hbp_attention_workspace_size(C.byref(d), C.byref(n))
    b = B.hbp_attention_buffers(C.sizeof(B.hbp_attention_buffers))
    for i, name in enumerate(("q", "k", "v", "o", "dout", "dq", "dk", "dv")):
        setattr(b, name, heads(A * (i + 1)))
    b.lse = A * 20
    b.workspace, b.workspace_bytes = A * 30, max(n.value, 1)
    for name, v in kw.items():
        setattr(b, name, v)
    return b


BAD = [(dict(struct_size=8), INVALID), (dict(q=heads(0)), NULL), (dict(k=heads(0)), NULL), (dict(v=heads(A + 8)), UNSUPPORTED),
       (dict(q=heads(row=1 << 24)), UNSUPPORTED), (dict(k=heads(head=4)), UNSUPPORTED), (dict(v=heads(row=-64)), INVALID), (dict(lse=0), NULL)]
BAD_FORWARD = [(dict(o=heads(0)), NULL), (dict(o=heads(row=64)), INVALID), (dict(o=heads(row=0, head=64)), INVALID)]
BAD_BACKWARD = [(dict(workspace=0), WORKSPACE), (dict(workspace_bytes=1), WORKSPACE), (dict(workspace=A * 30 + 4), UNSUPPORTED),
                (dict(dout=heads(0)), NULL), (dict(dq=heads(row=256, head=0)), INVALID), (dict(dk=heads(row=64, head=64)), INVALID),
                (dict(dv=heads(0)), NULL)]


@pytest.mark.parametrize("kw,status", BAD + BAD_FORWARD)
def test_attention_forward_refusals(kw, status):
    d = desc()
    assert B.lib().hbp_attention_forward(C.byref(d), C.byref(buffers(d, **kw)), None) == status


@pytest.mark.parametrize("kw,status", BAD + BAD_BACKWARD)
def test_attention_backward_refusals(kw, status):
    d = desc()
    assert B.lib().hbp_attention_backward(C.byref(d), C.byref(buffers(d, **kw)), None) == status


def test_attention_refuses_unequal_lengths_without_offsets_and_missing_structs():
    d = desc(q_rows=63)
    assert B.lib().hbp_attention_forward(C.byref(d), C.byref(buffers(d)), None) == INVALID
    assert B.lib().hbp_attention_forward(None, C.byref(buffers(desc())), None) == NULL
    assert B.lib().hbp_attention_forward(C.byref(desc()), None, None) == NULL
    assert B.lib().hbp_attention_workspace_size(C.byref(desc()), None) == NULL


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError):
        B.hbp_rotary(B.make_rotary(8), x, x)                                   # not on the GPU
    with pytest.raises(ValueError):
        B.hbp_rotary(B.make_rotary(8), x, torch.zeros(4, 2, 16))
    with pytest.raises(ValueError):
        B.hbp_rotary(B.make_rotary(8), x.transpose(1, 2), x.transpose(1, 2))   # channels apart
    with pytest.raises(ValueError):
        B.hbp_rotary(B.make_rotary(8), x, x, positions=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.hbp_rotary(B.make_rotary(8), x.half(), x.half())
    with pytest.raises(ValueError):
        B.make_attention(x, x, x)


TFM = dict(kind="transformer", dtype="bf16", act="gelu", norm="rms", L=4, N=64, d=128, d_ff=256, heads=4, seq_len=32)


def test_transformer_with_positions_and_shared_heads_descriptor_rules():
    n = C.c_size_t(0)
    size = lambda d: B.lib().hbp_workspace_size(C.byref(d), C.byref(n))
    full = B.make_desc(**TFM)
    assert size(full) == OK
    plain = n.value
    assert size(B.make_desc(**TFM, kv_heads=4)) == OK and n.value == plain
    assert size(B.make_desc(**TFM, kv_heads=4, rotary=B.make_rotary(32))) == OK and n.value == plain
    assert size(B.make_desc(**TFM, kv_heads=1)) == OK and 0 < n.value < plain + 4096
    for bad in (dict(kv_heads=3), dict(kv_heads=-1), dict(kv_heads=8), dict(rotary=B.make_rotary(34)), dict(rotary=B.make_rotary(3)),
                dict(rotary=B.make_rotary(32, base=-1.0))):
        assert size(B.make_desc(**TFM, **bad)) == INVALID, bad
    d = B.make_desc(**TFM, kv_heads=2)
    d.reserved = 1
    assert size(d) == INVALID
    d = B.make_desc(**dict(TFM, kind="mlp", heads=0, seq_len=0), kv_heads=2)
    assert size(d) == INVALID                                               # another kind has no such descriptor
    wide = dict(TFM, d=576, heads=4, d_ff=64)                                  # heads of 144 channels
    assert size(B.make_desc(**wide)) == OK and size(B.make_desc(**wide, kv_heads=2)) == UNSUPPORTED


def test_struct_sizes_match_header(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("hbp_rotary_desc", "hbp_heads", "hbp_attention_desc", "hbp_attention_buffers", "hbp_transformer_desc")
    src = tmp_path / "sizes.c"
    src.write_text('#include "hbp.h"\n#include <stdio.h>\nint main(void) {\n' +
                   "".join(f'  printf("%zu ", sizeof({n}));\n' for n in names) +
                   '  printf("%zu %zu", offsetof(hbp_transformer_desc, rotary), offsetof(hbp_attention_buffers, lse));\n  return 0;\n}\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(getattr(B, n)) for n in names] + [B.hbp_transformer_desc.rotary.offset, B.hbp_attention_buffers.lse.offset]


# ---- the reference ------------------------------------------------------------------------------------------------
def _problem(lq, lk, H, K, D, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    return r(sum(lq), H, D), r(sum(lk), K, D), r(sum(lk), K, D), r(sum(lq), H, D)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([3, 0, 5], [3, 2, 5]), ([4, 6], [7, 2])])
def test_reference_gradients_against_differences(lq, lk, causal):
    q, k, v, do = _problem(lq, lk, 4, 2, 8)
    value = lambda: (R.Packed(q, k, v, lq, lk, causal).forward()[0] * do).sum().item()
    o, lse, _, _ = R.Packed(q, k, v, lq, lk, causal).forward()
    grads = R.Packed(q, k, v, lq, lk, causal).backward(o, lse, do)[:3]
    for t, grad in zip((q, k, v), grads):
        for i in range(0, t.numel(), 7):
            flat = t.view(-1)
            keep = flat[i].item()
            flat[i] = keep + 1e-5
            up = value()
            flat[i] = keep - 1e-5
            down = value()
            flat[i] = keep
            assert abs((up - down) / 2e-5 - grad.flatten()[i].item()) < 1e-7      # h^2 f''' / 6 and 2^-52 |f| / h, both below 1e-8


@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=4.0),
                                     dict(scaling="by_parts", factor=4.0, original=64)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_reference_rotary(layout, scaling):
    """Inner products of turned rows depend on the distance of their positions alone; the inverse is the transpose."""
    x, _, _, y = _problem([6], [6], 2, 2, 16)
    pos = torch.tensor([0, 3, 4, 9, 100, 7])
    a, b = (R.rotary(t, p, 12, layout, **scaling)[0] for t, p in ((x, pos), (y, pos + 2)))
    c, d = (R.rotary(t, p, 12, layout, **scaling)[0] for t, p in ((x, pos + 31), (y, pos + 33)))
    assert torch.allclose((a * b).sum(-1), (c * d).sum(-1), rtol=0, atol=1e-12)
    back = R.rotary(y, pos, 12, layout, inverse=True, **scaling)[0]
    assert abs((a * y).sum() - (x * back).sum()) < 1e-12
    assert torch.equal(a[..., 12:], x[..., 12:]) and torch.equal(a[0], x[0])


def test_reference_notices_a_wrong_element():
    q, k, v, do = _problem([5], [5], 2, 1, 8)
    o, lse, eo, el = R.Packed(q.float(), k.float(), v.float(), [5], [5], True).forward()
    R.assert_within(o, o, eo, "itself")
    wrong = o.clone()
    wrong[3, 1, 2] += 1e-4
    with pytest.raises(AssertionError):
        R.assert_within(wrong, o, eo, "planted")
    wrong = o.clone()
    wrong[0, 0, 0] = math.nan
    with pytest.raises(AssertionError):
        R.assert_within(wrong, o, eo, "planted")


def test_a_tensor_that_is_not_there_is_refused():
    """An Attention made without room for gradients has no dq, dk, dv."""
    with pytest.raises(ValueError, match="dq: .* got none"):
        B._heads("dq", None, (4, 2, 8), torch.float32, 0)
