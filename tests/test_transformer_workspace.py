"""CPU-only: what a transformer stack with shared key/value heads reserves for its attention, against what the attention of any number of
its layers needs.  (The backward pass takes fewer and fewer layers at a time, and the need does not grow with their number.)"""
import ctypes as C

import pytest

from paper_2501_17086_amd import binding as B


def stack_bytes(dtype, L, N, T, heads, kv, dh):
    n = C.c_size_t(0)
    desc = B.make_desc(kind="transformer", dtype=dtype, act="gelu", norm="rms", L=L, N=N, d=heads * dh, d_ff=64, heads=heads, seq_len=T,
                       kv_heads=kv)
    assert B.lib().hbp_workspace_size(C.byref(desc), C.byref(n)) == 0
    return n.value


def attention_bytes(dtype, layers, N, T, heads, kv, dh):
    """Of `layers` layers' sequences behind one another."""
    return B.attention_workspace_size(B.hbp_attention_desc(
        C.sizeof(B.hbp_attention_desc), B.BF16 if dtype == "bf16" else B.F32, heads, kv, dh, 1, dh ** -0.5, 0.0, layers * (N // T),
        layers * N, layers * N))


def aligned(n):
    return (n + 255) // 256 * 256


def before_attention(dtype, L, N, heads, kv, dh):
    """Bytes of the stack's workspace before the attention's.  Sequences of 32 tokens with groups of up to four heads are too short
    to be shared out, so that there all layers together need most; nothing else depends on the sequences' length."""
    assert heads // kv <= 4 and N % 32 == 0
    return stack_bytes(dtype, L, N, 32, heads, kv, dh) - aligned(attention_bytes(dtype, L // 2, N, 32, heads, kv, dh))


# layers, tokens, tokens of a sequence, heads, key heads, channels of a head
KNOWN = [(16, 2048, 256, 4, 2, 64), (16, 2048, 64, 8, 2, 64), (34, 512, 128, 8, 4, 64), (12, 2048, 256, 16, 4, 64)]
GRID = [(L, S * T, T, K * G, K, dh) for L in (2, 8, 24, 48) for S in (1, 3, 8, 32) for T in (64, 96, 256, 480, 1024)
        for K, G in ((1, 2), (2, 2), (2, 4), (8, 4), (5, 3)) for dh in (64, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [KNOWN, GRID], ids=["known", "grid"])
def test_a_stack_reserves_what_any_number_of_its_layers_needs(sizes, dtype):
    for L, N, T, heads, kv, dh in sizes:
        reserved = stack_bytes(dtype, L, N, T, heads, kv, dh) - before_attention(dtype, L, N, heads, kv, dh)
        needs = [attention_bytes(dtype, n, N, T, heads, kv, dh) for n in range(1, L // 2 + 1)]
        assert reserved == aligned(max(needs)), (L, N, T, heads, kv, dh, reserved, max(needs), needs.index(max(needs)) + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_heads_reserve_nothing_for_the_attention_of_equal_heads(dtype):
    """Before the attention's own room a stack's workspace depends on the width of q, k, v alone, not on the number of heads."""
    for L, N in ((2, 64), (8, 4096)):
        a, b = before_attention(dtype, L, N, 8, 4, 32), before_attention(dtype, L, N, 4, 2, 64)
        assert a == b, (L, N)
