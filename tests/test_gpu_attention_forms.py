"""Every form of the attention over packed sequences on the GPU, at head widths, layouts and lengths where forms differ: against the
definitions in 64 bits (tests/attention_reference.py derives the bounds), or bit by bit against the same values laid out otherwise."""
import math

import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import attention_reference as R
from tests.test_gpu_attention_ops import FORMS, SENTINEL, TALL, check_attention, offsets, problem, strided

pytestmark = pytest.mark.gpu
NAMES = ("o", "lse", "dq", "dk", "dv")


def sizes(form, dh):
    """As test_attention_forms takes them: fewer heads where the reference would take long."""
    lq, lk, H, K = form
    lk = lq if lk is None else lk
    return (lq, lk, H // K, 1) if len(lq) * max(lq) * max(lk) * H * dh > 3e10 else (lq, lk, H, K)


# indexes into FORMS: bf16 wavefronts by themselves, workgroups of many rows (keys), of few, with and without shares; fp32 of 128 rows with
# and without shares, of 32
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form,dh", [(f, dh) for f in (2, 3, 5, 6, 7, 9) for dh in (32, 96)] + [(f, dh) for f in (2, 6) for dh in (24, 40, 88, 104)])
def test_widths_in_every_form(form, dh, dtype):
    lq, lk, H, K = sizes(FORMS[form], dh)
    q, k, v, do = problem(lq, lk, H, K, dh, dtype, 211)
    for causal in (True, False):
        check_attention(q, k, v, lq, lk, causal, do)


def run(q, k, v, do, off, how=None):
    """Outputs of a call on these values, laid out as `how` says; nothing between them is written."""
    a = B.make_attention(q, k, v, **off)
    around = {}
    for name in ("o", "dq", "dk", "dv"):
        t = torch.full_like(getattr(a, name), SENTINEL)
        around[name], view = (t, t) if how is None else strided(t, how)
        setattr(a, name, view)
    a.lse.fill_(SENTINEL)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    out = {name: getattr(a, name).clone() for name in NAMES}
    for name, big in around.items():
        getattr(a, name).fill_(SENTINEL)
        assert bool((big == SENTINEL).all()), f"{name}: written outside"
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["rows", "heads"])
@pytest.mark.parametrize("dh", [64, 96])
@pytest.mark.parametrize("form", range(len(FORMS) + 1))
def test_strides_in_every_form(form, dh, how, dtype):
    lq, lk, H, K = (FORMS + TALL[1:2])[form]
    lk = lq if lk is None else lk
    t = problem(lq, lk, H, K, dh, dtype, 223)
    off = dict(q_offsets=offsets(lq), k_offsets=offsets(lk))
    want, got = run(*t, off), run(*(strided(x, how)[1] for x in t), off, how)
    for name in NAMES:
        assert torch.equal(want[name], got[name]), name


# one long sequence among many short ones, and short ones, empty ones included, among long ones
TAILS = [([3000] + [64] * 120, 4, 2), ([7, 0, 900] + [5] * 300 + [1700], 4, 1), ([2000, 0, 1, 5, 64, 33, 700] * 3, 32, 8),
         ([700, 0, 1, 5, 64, 33, 300] * 6, 8, 4), ([1] * 100 + [2500], 2, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lens,H,K", TAILS, ids=[f"{len(t[0])}of{max(t[0])}" for t in TAILS])
def test_lengths_far_from_their_mean(lens, H, K, dh, dtype):
    q, k, v, do = problem(lens, lens, H, K, dh, dtype, 227)
    check_attention(q, k, v, lens, lens, True, do)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_rows_of_nothing_in_every_form(form, dtype):
    """Keys that all score minus infinity in the first sequence: its rows weigh nothing and pass no gradient on, in dv and dk neither.  The
    other sequences are as with the sequence's keys finite."""
    lq, lk, H, K = sizes(FORMS[form], 64)
    q, k, v, do = problem(lq, lk, H, K, 64, dtype, 229)
    q[:lq[0], :, 0] = 1.0
    off = dict(q_offsets=offsets(lq), k_offsets=offsets(lk), causal=False)
    want = run(q, k, v, do, off)
    k[:lk[0], :, 0] = -math.inf
    got = run(q, k, v, do, off)
    n, m = lq[0], lk[0]
    assert bool((got["lse"][:n] == -math.inf).all()) and not got["o"][:n].any()
    assert not got["dv"][:m].any()
    for name, first in (("o", n), ("lse", n), ("dq", n), ("dk", m), ("dv", m)):
        assert torch.equal(want[name][first:], got[name][first:]), name


# ragged on one side, of equal lengths on the other: few sequences, and more than are searched one by one
MIXED = [([3, 0, 17, 90], 64), ([300, 1, 520], 700), ([i % 5 for i in range(200)], 33), ([40 + i % 9 for i in range(140)], 8), ([1900], 1200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,each", MIXED, ids=[f"{len(m[0])}of{max(m[0])}x{m[1]}" for m in MIXED])
def test_offsets_on_one_side_alone(lens, each, causal, dtype):
    """As with the equal lengths spelt out on the other side."""
    for lq, lk in ((lens, [each] * len(lens)), ([each] * len(lens), lens)):
        q, k, v, do = problem(lq, lk, 4, 2, 64, dtype, 233)
        off = dict(q_offsets=offsets(lq), k_offsets=offsets(lk), causal=causal)
        want = run(q, k, v, do, off)
        off["k_offsets" if lq is lens else "q_offsets"] = None
        got = run(q, k, v, do, off)
        for name in NAMES:
            assert torch.equal(want[name], got[name]), name
        if len(lens) < 10:
            check_attention(q, k, v, lq, lk, causal, do)
