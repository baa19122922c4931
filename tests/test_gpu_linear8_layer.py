"""A decoder layer whose projections and whose cache are in 8 bits, every call on what the one before it gave."""
import numpy as np
import pytest
import torch

from linear8_testlib import U, check_product, check_rows, gate_and_up, random_rows, row_values
from test_gpu_kvquant import HD, check_attend, cu_of, make_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
D, FFN, HEADS, KV = 384, 512, 6, 2
EPS = 2.0 ** -16   # (a float)


class Layer:
    def __init__(self, scale):
        from paper_2602_12957_amd import linear8 as L
        self.L = L
        make = lambda n, k, seed: L.Weight8.quantize(random_rows(n, k, seed, spread=0.2) / k ** 0.5, scale)   # noqa: E731
        self.qkv, self.o = make((HEADS + 2 * KV) * HD, D, 1), make(D, HEADS * HD, 2)
        self.gate_up, self.down = make(2 * FFN, D, 3), make(D, FFN, 4)
        self.gains = 1 + 0.1 * random_rows(2, D, 5, F32, spread=0.0)

    def step(self, cache, cu, delta, res):
        """One pass: all that its calls give, in their order."""
        L, n = self.L, len(delta)
        a, h = L.norm_rows(delta, self.gains[0], EPS, residual=res)
        qkv = L.linear(a, self.qkv)
        q, k, v = (t.view(n, -1, HD) for t in qkv.split([HEADS * HD, KV * HD, KV * HD], 1))
        slots, _ = cache.reserve(cu, n)
        cache.append(k, v, slots)
        att = cache.attend(q, cu)
        att8 = L.quantize_rows(att.view(n, HEADS * HD))
        o = L.linear(att8, self.o)
        b, h2 = L.norm_rows(o, self.gains[1], EPS, residual=h)
        u = L.gated(b, self.gate_up)
        return dict(a=a, h=h, qkv=qkv, slots=slots, att=att, att8=att8, o=o, b=b, h2=h2, u=u, out=L.linear(u, self.down))


def check_norm(rows8, total, x, res, gain):
    h = x.double() + res.double()
    assert bool(((total.double() - h).abs() <= U * h.abs()).all())
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS) * gain.double()
    check_rows(rows8, y, (D + 60) * 2.0 ** -53 * y.abs() + 2.0 ** -149)


@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_a_layer_from_prefill_to_single_tokens(scale):
    """Two sequences: prompts that end inside of pages, single tokens, a draft of which one sequence keeps two rows and the other none."""
    layer, cache = Layer(scale), make_cache(24, KV, 2, 12, shuffle=3)
    lens = np.zeros(2, np.int64)
    for step, (q, accept) in enumerate([([37, 90], None), ([1, 1], None), ([1, 1], None), ([5, 7], [1, -1]), ([1, 1], None)]):
        n, cu = sum(q), cu_of(q)
        delta, res = random_rows(n, D, 10 + step), random_rows(n, D, 20 + step, F32)
        r = layer.step(cache, cu, delta, res)
        check_norm(r["a"], r["h"], delta, res, layer.gains[0])
        check_product(r["qkv"], r["a"], layer.qkv)
        x = r["qkv"][:, :HEADS * HD].reshape(n, HEADS, HD)
        check_attend(cache, r["att"], x, lens, q, BF)
        check_rows(r["att8"], r["att"].reshape(n, HEADS * HD).double(), 0.0)
        check_product(r["o"], r["att8"], layer.o)
        check_norm(r["b"], r["h2"], r["o"], r["h"], layer.gains[1])
        want, worst, _ = gate_and_up(r["b"], layer.gate_up)
        check_rows(r["u"], want, worst)
        check_product(r["out"], r["u"], layer.down)
        if accept is None:
            cache.commit(cu, n)
            lens += q
        else:
            cache.commit(cu, n, torch.tensor(accept, dtype=torch.int32, device=DEV))
            lens += [2, 0]
        np.testing.assert_array_equal(cache.seq_len.cpu().numpy(), lens)
    assert int(cache.status.item()) == 0


def test_a_captured_layer_replays():
    """A step of single tokens in one graph, replayed on new rows with eager passes between."""
    layer, cache = Layer(torch.uint8), make_cache(24, KV, 2, 12, shuffle=3)
    cu, n = cu_of([37, 90]), 127
    layer.step(cache, cu, random_rows(n, D, 1), random_rows(n, D, 2, F32))
    cache.commit(cu, n)
    cache.snapshot()
    cu, delta, res = cu_of([1, 1]), random_rows(2, D, 3), random_rows(2, D, 4, F32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(cache, cu, delta, res)
    torch.cuda.current_stream().wait_stream(side)
    cache.restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = layer.step(cache, cu, delta, res)
    same = lambda p, q: torch.equal(row_values(p.codes, p.scale, p.dim), row_values(q.codes, q.scale, q.dim)) if hasattr(p, "codes") else torch.equal(p, q)   # noqa: E731
    for rep in range(4):
        delta.copy_(random_rows(2, D, 30 + rep)), res.copy_(random_rows(2, D, 40 + rep, F32))
        cache.restore()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: (type("R", (), dict(codes=v.codes.clone(), scale=v.scale.clone(), dim=v.dim)) if hasattr(v, "codes") else v.clone()) for k, v in kept.items()}
        cache.restore()
        want = layer.step(cache, cu, delta, res)
        torch.cuda.synchronize()
        assert all(same(got[k], want[k]) for k in got), rep
