"""The conditioned block's attention as it is used: query, key and value projections with the requests' adapters, cross attention to an encoder's
states, the output projection with adapters, forward and backward, eager, on another stream and in captured graphs."""
import math

import pytest
import torch

from paper_2511_20390_amd import binding as b
from tests.block_ops_util import check
from tests.cond_ops_util import adapters_reference, cross_reference, keys_that_count

pytestmark = pytest.mark.gpu

DEV = "cuda"
MODE = {torch.bfloat16: "bf16", torch.float32: "fp32"}


class Block:
    """B samples of Nq tokens of width D that attend to Nk states of width E; every projection has adapters of rank r."""

    def __init__(self, seed, dtype, B, Nq, Nk, heads, kv, dh, D, E, r, n):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        normal = lambda shape, std: torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0, std, generator=gen).to(dtype)
        self.B, self.Nq, self.Nk, self.heads, self.kv, self.dh = B, Nq, Nk, heads, kv, dh
        self.x, self.states, self.g = normal((B * Nq, D), 1.0), normal((B * Nk, E), 1.0), normal((B * Nq, D), 1.0)
        # (input width, output width, rows of a sample)
        self.layers = {"q": (D, heads * dh, Nq), "kv": (E, 2 * kv * dh, Nk), "o": (heads * dh, D, Nq)}
        self.w = {name: normal((N, K), K ** -0.5) for name, (K, N, _) in self.layers.items()}
        self.a = {name: normal((n, r, K), K ** -0.5) for name, (K, N, _) in self.layers.items()}
        self.b = {name: normal((n, N, r), r ** -0.5) for name, (K, N, _) in self.layers.items()}
        self.bias = {name: torch.empty(N, device=DEV).normal_(0, 1, generator=gen) for name, (K, N, _) in self.layers.items()}
        self.adapter = torch.randint(-1, n, (B,), device=DEV, dtype=torch.int32, generator=gen)
        self.scale = 0.5 + torch.rand(n, device=DEV, generator=gen)
        self.key_len = torch.randint(1, Nk + 1, (B,), device=DEV, dtype=torch.int32, generator=gen)
        mode, M = MODE[dtype], {name: B * rows for name, (_, _, rows) in self.layers.items()}
        byte = lambda k: torch.empty(k, dtype=torch.uint8, device=DEV)
        self.saved = {name: byte(b.linear_adapters_saved_bytes(M[name], r, mode)) for name in self.layers}
        # one workspace for all of them, which come one after the other on a stream
        self.ws = byte(max([b.linear_adapters_workspace_bytes(M[name], K, N, r, n, mode, backward=True) for name, (K, N, _) in self.layers.items()] +
                           [b.cross_attention_workspace_bytes(B, Nq, Nk, heads, kv, dh, mode, backward=True)]))
        self.lse = torch.empty(B, heads, Nq, device=DEV)

    def _linear(self, name, x):
        return b.op_linear_adapters(x, self.w[name], self.bias[name], self.a[name], self.b[name], self.adapter, scale=self.scale,
                                    rows_per_sample=self.layers[name][2], saved=self.saved[name], workspace=self.ws)

    def _linear_back(self, name, g, x):
        return b.op_linear_adapters_backward(g, x, self.w[name], self.a[name], self.b[name], self.adapter, self.saved[name], scale=self.scale,
                                             rows_per_sample=self.layers[name][2], workspace=self.ws)

    def run(self):
        """All tensors between the operators, and the gradients, by name."""
        how = dict(B=self.B, heads=self.heads, dh=self.dh, kv_heads=self.kv, key_len=self.key_len, workspace=self.ws)
        half = self.kv * self.dh
        t = {"q": self._linear("q", self.x), "kv": self._linear("kv", self.states)}
        k, v = t["kv"][:, :half], t["kv"][:, half:]
        t["att"] = b.op_cross_attention(t["q"], k, v, lse=self.lse, **how)
        t["out"] = self._linear("o", t["att"])
        t["datt"], t["da_o"], t["db_o"] = self._linear_back("o", self.g, t["att"])
        t["dkv"] = torch.empty_like(t["kv"])
        t["dq"], _, _ = b.op_cross_attention_backward(t["datt"], t["q"], k, v, t["att"], self.lse, **how,
                                                      grads=(torch.empty_like(t["q"]), t["dkv"][:, :half], t["dkv"][:, half:]))
        t["dx"], t["da_q"], t["db_q"] = self._linear_back("q", t["dq"], self.x)
        t["dstates"], t["da_kv"], t["db_kv"] = self._linear_back("kv", t["dkv"], self.states)
        return t

    def check(self, t):
        """Each operator against the formula in 64 bits of what it was given."""
        half = self.kv * self.dh

        def linear(name, x, g, outs):
            ref = adapters_reference(x, self.w[name], self.bias[name], self.a[name], self.b[name], self.adapter, self.scale, self.layers[name][2], g)
            for key, r in zip(outs, ref):
                check(t[key], r, key)

        linear("q", self.x, t["dq"], ("q", "dx", "da_q", "db_q"))
        linear("kv", self.states, t["dkv"], ("kv", "dstates", "da_kv", "db_kv"))
        linear("o", t["att"], self.g, ("out", "datt", "da_o", "db_o"))
        k, v = t["kv"][:, :half], t["kv"][:, half:]
        keys = keys_that_count(self.B, self.Nk, self.key_len, None, DEV)
        ref = cross_reference(t["q"], k, v, self.B, self.heads, self.kv, self.dh, self.dh ** -0.5, keys, t["datt"])
        for got, r, what in ((t["att"], ref[0], "att"), (self.lse, ref[1], "lse"), (t["dq"], ref[2], "dq"), (t["dkv"][:, :half], ref[3], "dk"), (t["dkv"][:, half:], ref[4], "dv")):
            check(got, r, what)


SHAPES = [
    dict(B=3, Nq=50, Nk=33, heads=4, kv=2, dh=24, D=96, E=80, r=5, n=2),
    dict(B=4, Nq=256, Nk=77, heads=4, kv=4, dh=72, D=288, E=256, r=16, n=3),
    dict(B=8, Nq=1, Nk=300, heads=8, kv=2, dh=64, D=512, E=256, r=16, n=4),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_block(dtype, shape):
    block = Block(1, dtype, **shape)
    block.check(block.run())


@pytest.mark.parametrize("shape", SHAPES[:2])
def test_block_gradient_by_autograd(shape):
    """The chain of the operators' gradients against that of the plain formulas in 64 bits.  A value passes up to seven operators, each of which is off by
    its bound relative to sums of the values' sizes; the chain's limit is a thousand roundings of fp32 relative to the largest gradient, sums of
    up to 1024 values of its size growing like their root."""
    block = Block(2, torch.float32, **shape)
    t = block.run()
    leaf = lambda v: v.double().detach().requires_grad_()
    x, states = leaf(block.x), leaf(block.states)
    a, bb = {k: leaf(v) for k, v in block.a.items()}, {k: leaf(v) for k, v in block.b.items()}

    def linear(name, v):
        rows = block.layers[name][2]
        which = block.adapter.long().repeat_interleave(rows)
        on = (which >= 0).double()[:, None] * block.scale.double()[which.clamp(min=0)][:, None]
        extra = torch.zeros(v.shape[0], bb[name].shape[1], dtype=torch.float64, device=DEV)
        for i in range(a[name].shape[0]):
            at = (which == i).double()[:, None]
            extra = extra + at * on * ((v @ a[name][i].T) @ bb[name][i].T)
        return v @ block.w[name].double().T + block.bias[name].double() + extra

    B, heads, kv, dh = block.B, block.heads, block.kv, block.dh
    per_head = lambda v, n: v.reshape(B, -1, n, dh).transpose(1, 2)
    q, kvs = linear("q", x), linear("kv", states)
    share = lambda v: per_head(v, kv).repeat_interleave(heads // kv, dim=1)
    s = per_head(q, heads) @ share(kvs[:, :kv * dh]).transpose(2, 3) * dh ** -0.5
    keys = keys_that_count(B, block.Nk, block.key_len, None, DEV)
    p = torch.softmax(s.masked_fill(~keys[:, None, None, :], -math.inf), dim=3)
    att = (p @ share(kvs[:, kv * dh:])).transpose(1, 2).reshape(B * block.Nq, heads * dh)
    (linear("o", att) * block.g.double()).sum().backward()
    for key, want in (("dx", x), ("dstates", states), ("da_q", a["q"]), ("db_q", bb["q"]), ("da_kv", a["kv"]), ("db_kv", bb["kv"]), ("da_o", a["o"]), ("db_o", bb["o"])):
        r = want.grad
        assert (t[key].double() - r).abs().max().item() <= 1000 * 2.0 ** -24 * r.abs().max().item(), key


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_another_stream(dtype):
    block = Block(3, dtype, **SHAPES[1])
    want = block.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = block.run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[k], got[k]) for k in want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_graphs_share_a_workspace(dtype):
    """Two blocks, captured one after the other with one workspace, replayed in turn with other inputs and eager calls between."""
    one, two = Block(4, dtype, **SHAPES[1]), Block(5, dtype, **SHAPES[0])
    two.ws = one.ws = max(one.ws, two.ws, key=torch.Tensor.numel)
    for block in (one, two):
        block.run()
    torch.cuda.synchronize()
    graphs, results = [], []
    for block in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(block.run())
        graphs.append(graph)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    for k in range(4):
        for block, graph, result in zip((one, two), graphs, results):
            for t in (block.x, block.states, block.g):
                t.copy_(torch.randn(t.shape, device=DEV, generator=gen))
            block.adapter.copy_(torch.roll(block.adapter, 1))
            block.key_len.copy_(torch.randint(0, block.Nk + 1, (block.B,), device=DEV, dtype=torch.int32, generator=gen))
            want = block.run()
            graph.replay()
            assert all(torch.equal(want[key], result[key]) for key in want), k
    one.check(results[0])


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own."""
    blocks = [Block(7 + i, torch.bfloat16, **SHAPES[1]) for i in range(2)]
    want = [block.run() for block in blocks]
    streams = [torch.cuda.Stream() for _ in blocks]
    got = []
    for block, s in zip(blocks, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(block.run())
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(w[k], g[k]) for w, g in zip(want, got) for k in w)
