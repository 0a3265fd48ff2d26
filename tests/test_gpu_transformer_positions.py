"""Transformer stacks with rotary positions and shared key/value heads on the GPU: forward states, exact and iterated state
gradients and all parameter gradients against the stack written out in torch operations of 64 bits on the CPU."""
import math

import numpy as np
import pytest
import torch

from paper_2501_17086_amd import binding as B, synth
from tests import attention_reference as R
from tests.helpers import TOL, assert_close, to_np

pytestmark = pytest.mark.gpu


class Stack:
    """Pre-norm layers, attention and feed-forward sub-blocks in turn, in 64 bits."""

    def __init__(self, w, inp, positions):
        t = lambda a: None if a is None else torch.from_numpy(np.asarray(a)).double()
        self.w, self.pos = w, positions
        self.W = {n: t(inp[n]).requires_grad_() for n in ("Wqkv", "Wo", "W1", "W2")}
        self.lam = t(inp["lam"]) if inp["lam"] is not None else torch.ones(w.L, w.d, dtype=torch.float64)
        self.x0, self.e = t(inp["x0"]), t(inp["e"])

    def block(self, l, x):
        w, j = self.w, l // 2
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + w.eps)
        if l % 2:
            return torch.nn.functional.gelu(y @ self.W["W1"][j].T) @ self.W["W2"][j].T
        H, K, D = w.heads, w.kv_heads or w.heads, w.d // w.heads
        qkv = (y @ self.W["Wqkv"][j].T).view(-1, H + 2 * K, D)
        if w.rotary:
            r = dict(w.rotary)
            qkv = torch.cat((self.turn(qkv[:, :H + K], r.pop("dims"), r.pop("layout", "half"), r.pop("magnitude", 1.0), r), qkv[:, H + K:]), 1)
        qkv = qkv.view(-1, w.seq_len, H + 2 * K, D).transpose(1, 2)
        q, k, v = qkv[:, :H], qkv[:, H:H + K].repeat_interleave(H // K, 1), qkv[:, H + K:].repeat_interleave(H // K, 1)
        s = q @ k.transpose(2, 3) / math.sqrt(D)
        if w.causal:
            s = s.masked_fill(torch.ones(w.seq_len, w.seq_len).triu(1).bool(), -math.inf)
        o = (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(x.shape)
        return o @ self.W["Wo"][j].T

    def turn(self, x, dims, layout, magnitude, scaling):
        t = torch.outer(self.pos.double(), R.frequencies(dims, **scaling))[:, None]
        c, s = torch.cos(t) * magnitude, torch.sin(t) * magnitude
        h = dims // 2
        a, b = (x[..., :h], x[..., h:dims]) if layout == "half" else (x[..., 0:dims:2], x[..., 1:dims:2])
        u, v = a * c - b * s, a * s + b * c
        both = torch.cat((u, v), -1) if layout == "half" else torch.stack((u, v), -1).flatten(-2)
        return torch.cat((both, x[..., dims:]), -1)

    def run(self):
        self.x = [self.x0.clone().requires_grad_()]
        for l in range(self.w.L):
            self.x.append(self.lam[l] * self.x[-1] + self.block(l, self.x[-1]))
        return self.x

    def exact(self):
        x = self.run()
        return torch.stack(torch.autograd.grad((x[-1] * self.e).sum(), x))

    def vjp(self, l, g):
        x = self.x[l].detach().requires_grad_()
        return torch.autograd.grad((self.block(l, x) * g).sum(), x)[0]

    def iterate(self, k, gamma):
        L, lam = self.w.L, self.lam
        g = [None] * L + [self.e]
        for it in range(k + 1):
            old = list(g)
            for l in range(L - 1, -1, -1):
                if it == 0:
                    g[l] = (1 - gamma) * lam[l] * g[l + 1]
                else:
                    g[l] = self.vjp(l, old[l + 1]) + gamma * lam[l] * old[l + 1] + (1 - gamma) * lam[l] * g[l + 1]
        return torch.stack(g)

    def param_grads(self, g):
        total = sum((self.block(l, self.x[l].detach()) * g[l + 1]).sum() for l in range(self.w.L))
        return dict(zip(self.W, torch.autograd.grad(total, list(self.W.values()))))


BASE = synth.scaled(synth.WORKLOADS["gpt2_paper"], name="positions", L=4, N=160, seq_len=40, d=128, heads=4, d_ff=256, w1_std=0.0,
                    w2_std=0.0, w2_scale=0.6)
CASES = {
    "shared": dict(kv_heads=2, rotary=dict(dims=32)),
    "one_key_head": dict(kv_heads=1, rotary=dict(dims=12, layout="interleaved", scaling="by_parts", factor=4.0, original=20.0, magnitude=1.1),
                         causal=False),
    "equal_heads": dict(rotary=dict(dims=32, base=500.0), seq_len=80),
    "no_positions": dict(kv_heads=2, d=192, heads=6, seq_len=32, lam="uniform", lam_lo=0.9, lam_hi=1.0),
    "wide_heads": dict(kv_heads=1, heads=2, d=256, rotary=dict(dims=64), seq_len=160, L=2),
}


def make(case, dtype, **kw):
    w = synth.scaled(BASE, **dict(dict(dtype=dtype), **CASES[case]), **kw)
    inp = synth.make_inputs(w)
    return w, inp, B.allocate(w, inp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", list(CASES))
def test_stack(case, dtype):
    w, inp, p = make(case, dtype)
    st = Stack(w, inp, torch.arange(w.N) % w.seq_len)
    exact = st.exact().detach().numpy()
    B.hbp_forward(p)
    assert_close(to_np(p.x), torch.stack(st.x).detach().numpy(), TOL[dtype], "x")
    B.hbp_exact_backward(p)
    assert_close(to_np(p.g), exact, TOL[dtype], "exact g")
    B.hbp_param_grads(p)
    for n, want in st.param_grads(torch.from_numpy(exact)).items():
        assert_close(to_np(getattr(p, "d" + n)), want.detach().numpy(), TOL[dtype], "d" + n)
    for k, gamma in ((0, 0.2), (1, 0.0), (2, 0.2), (w.L, 0.2)):
        B.hbp_backward(p, k, gamma=gamma)
        assert_close(to_np(p.g), st.iterate(k, gamma).detach().numpy(), TOL[dtype], f"g k={k} gamma={gamma}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_given_positions(dtype):
    """Documents that do not start with a sequence: every token's position is its own."""
    w, inp, p = make("shared", dtype)
    pos = (torch.arange(w.N) * 7) % 53
    given = pos.to(torch.int32).cuda()
    p.desc.positions = given.data_ptr()
    st = Stack(w, inp, pos)
    exact = st.exact().detach().numpy()
    B.hbp_forward(p)
    assert_close(to_np(p.x), torch.stack(st.x).detach().numpy(), TOL[dtype], "x")
    B.hbp_exact_backward(p)
    assert_close(to_np(p.g), exact, TOL[dtype], "exact g")
    B.hbp_backward(p, w.L)
    assert_close(to_np(p.g), exact, TOL[dtype], "g k=L")


def test_without_either_the_descriptor_changes_nothing():
    w, inp, p = make("equal_heads", "bf16")
    plain = B.allocate(synth.scaled(w, rotary=None), inp)
    p.desc.rotary = B.hbp_rotary_desc()
    for x in (p, plain):
        B.hbp_forward(x)
        B.hbp_backward(x, 2)
        B.hbp_param_grads(x)
    for n in ("x", "g", "qkv", "attn_o", "lse", "dWqkv", "dWo", "dW1", "dW2"):
        assert torch.equal(getattr(p, n), getattr(plain, n)), n


@pytest.mark.parametrize("case", ["shared", "equal_heads"])
def test_training_step_is_its_parts_and_a_graph_replays_them(case):
    w, inp, p = make(case, "bf16")
    target = torch.zeros_like(p.x[-1])
    opt = B.make_optim("adamw", 1e-3)
    keep = {n: getattr(p, n).clone() for n in ("W1", "W2", "Wqkv", "Wo")}
    B.hbp_train_step(p, 2, target, opt, B.allocate_optim(p, adamw=True))
    after = {n: getattr(p, n).clone() for n in list(keep) + ["dWqkv", "dWo", "g"]}
    for n, t in keep.items():
        getattr(p, n).copy_(t)
    st = B.allocate_optim(p, adamw=True)
    B.hbp_forward(p)
    B.hbp_loss_mse(p, target, st)
    B.hbp_backward(p, 2)
    B.hbp_param_grads(p)
    for n in ("dWqkv", "dWo", "g"):
        assert torch.equal(getattr(p, n), after[n]), n
    B.hbp_optimizer_step(p, opt, st)
    for n in keep:
        assert torch.equal(getattr(p, n), after[n]), n
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.hbp_forward(p)
        B.hbp_backward(p, 2)
        B.hbp_param_grads(p)
    B.hbp_forward(p)
    B.hbp_backward(p, 2)
    B.hbp_param_grads(p)
    want = (p.g.clone(), p.dWqkv.clone())
    for _ in range(3):
        p.g.zero_()
        p.dWqkv.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.g, want[0]) and torch.equal(p.dWqkv, want[1])
        B.hbp_backward(p, 0)


class PostNorm(Stack):
    """Layers without a norm before a sub-block, and one after every residual sum."""

    def block(self, l, x):
        w, j = self.w, l // 2
        if l % 2:
            return torch.nn.functional.gelu(x @ self.W["W1"][j].T) @ self.W["W2"][j].T
        H, K, D = w.heads, w.kv_heads, w.d // w.heads
        qkv = (x @ self.W["Wqkv"][j].T).view(-1, H + 2 * K, D)
        qkv = torch.cat((self.turn(qkv[:, :H + K], w.rotary["dims"], "half", 1.0, {}), qkv[:, H + K:]), 1)
        qkv = qkv.view(-1, w.seq_len, H + 2 * K, D).transpose(1, 2)
        q, k, v = qkv[:, :H], qkv[:, H:H + K].repeat_interleave(H // K, 1), qkv[:, H + K:].repeat_interleave(H // K, 1)
        o = torch.softmax(q @ k.transpose(2, 3) / math.sqrt(D), -1) @ v
        return o.transpose(1, 2).reshape(x.shape) @ self.W["Wo"][j].T

    def run(self):
        self.x = [self.x0.clone()]
        for l in range(self.w.L):
            s = self.lam[l] * self.x[-1] + self.block(l, self.x[-1])
            self.x.append(s / torch.sqrt((s * s).mean(-1, keepdim=True) + self.w.eps))
        return self.x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_post_norm_stack(dtype):
    """As the other stacks, where the norm follows the residual sum: states, and the exact gradients of all parameters."""
    w = synth.scaled(synth.WORKLOADS["roberta_like"], name="positions_post", dtype=dtype, L=4, N=120, seq_len=40, d=128, heads=4, d_ff=256,
                     w1_std=0.0, w2_std=0.0, w2_scale=0.6, kv_heads=2, rotary=dict(dims=32))
    inp = synth.make_inputs(w)
    p = B.allocate(w, inp)
    st = PostNorm(w, inp, torch.arange(w.N) % w.seq_len)
    x = st.run()
    want = dict(zip(st.W, torch.autograd.grad((x[-1] * st.e).sum(), list(st.W.values()))))
    B.hbp_forward(p)
    assert_close(to_np(p.x), torch.stack(x).detach().numpy(), TOL[dtype], "x")
    B.hbp_exact_backward(p)
    B.hbp_param_grads(p)
    for n, t in want.items():
        assert_close(to_np(getattr(p, "d" + n)), t.detach().numpy(), TOL[dtype], "d" + n)
