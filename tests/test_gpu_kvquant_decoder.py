"""The decoder's passes on an 8-bit cache against the fp64 oracle, which attends to the values that the engine's pages hold.

What the pages hold is compared on its own: a stored value is off by half a step of e4m3 (2^-4 of it, or 2^-10 of the scale where that
is more) for its own rounding and by 2^-10 of a scale for each later pass that raised the scale of its page, beyond what a pass in
the model's type leaves (the bars that hold for logits: 1e-4 in fp32, 2e-2 in bf16, of the layer's largest value or 1).
"""
import numpy as np
import pytest
import torch

import oracle as O
import workloads as W
import paper_2602_12957_amd.binding as B
from workloads.generators import SequenceSpec

from hsd_testlib import MARGIN_GATE, gated_compare_argmax, prefix_rows

pytestmark = pytest.mark.gpu

TOL = {"fp32": 1e-4, "bf16": 2e-2}
MODELS = {"fp32": W.ModelDesc(n_layers=2, d_model=128, n_q_heads=4, n_kv_heads=1, head_dim=64, d_ffn=256, vocab=512, dtype="fp32"),
          "bf16": W.ModelDesc(n_layers=3, d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ffn=512, vocab=1024, dtype="bf16")}


def make_engine(desc, weights, n_slots, maxb, max_q, n_blocks=None, **kw):
    from paper_2602_12957_amd.runtime import Engine
    return Engine(desc, weights, n_blocks or n_slots * min(maxb, 32), n_slots, maxb, max_q, kw.pop("max_dump", max_q), kv_cache="fp8", **kw)


def held_pages(eng, desc):
    """What the engine's pages hold: K, V [layer][block][head][token][dim] in fp64, and the scales [2][layer][block][head]."""
    L, H = desc.n_layers, desc.n_kv_heads
    out, scales = [], []
    for codes, scale, key in ((eng.k_pool, eng.k_scale, True), (eng.v_pool, eng.v_scale, False)):
        x = codes.cpu().view(torch.float8_e4m3fn).to(torch.float32).numpy().astype(np.float64).reshape(L, -1, H, 1024)
        s = scale.cpu().numpy().astype(np.float64)
        i = np.arange(1024)
        if key:      # [dims 16 g ..][token][16 dims]
            tok, dim = i // 16 % 16, 16 * (i // 256) + i % 16
        else:        # [half][pair of dims r][dim][8 tokens of the half]
            j = i % 8
            tok, dim = 8 * (j >> 2) + 4 * (i // 512) + (j & 3), 2 * (i // 16 % 32) + i // 8 % 2
        page = np.empty(x.shape[:3] + (16, 64))
        page[..., tok, dim] = x
        out.append(page * s[..., None, None])
        scales.append(s)
    return out[0], out[1], np.stack(scales)


class EngineCache(O.KVCache):
    """A sequence's history as the engine's pages hold it; rows written by the oracle are compared with it."""

    def __init__(self, eng, desc, slot):
        super().__init__(desc.n_layers, desc.n_kv_heads, desc.head_dim)
        self.eng, self.desc, self.slot, self.passes, self.top = eng, desc, slot, 0, None

    def look(self):
        """takes the pages of the pass that the engine has made"""
        k, v, s = held_pages(self.eng, self.desc)
        table = self.eng.block_table[self.slot].cpu().numpy()
        table = table[table >= 0]
        L, H = self.desc.n_layers, self.desc.n_kv_heads
        self.k, self.v = (x[:, table].transpose(0, 1, 3, 2, 4).reshape(L, -1, H, 64) for x in (k, v))
        s = s[:, :, table].repeat(16, axis=2)
        if self.top is not None:
            n = min(self.top.shape[2], s.shape[2])
            s[:, :, :n] = np.maximum(s[:, :, :n], self.top[:, :, :n])
        self.top = s
        self.passes += 1

    def keys(self, layer, n):
        return self.k[layer, :n]

    def values(self, layer, n):
        return self.v[layer, :n]

    def write(self, layer, pos0, k, v):
        n = pos0 + len(k)
        for got, ref, s in ((self.k, k, self.top[0]), (self.v, v, self.top[1])):
            bar = TOL[self.desc.dtype] * max(1.0, np.abs(ref).max())
            tol = bar + np.maximum(2.0 ** -4 * (np.abs(ref) + bar), 2.0 ** -10 * s[layer, pos0:n, :, None]) + self.passes * 2.0 ** -10 * s[layer, pos0:n, :, None]
            err = np.abs(got[layer, pos0:n] - ref)
            assert (err <= tol).all(), (layer, float((err / tol).max()))


def prefill(eng, desc, weights, seed, specs):
    toks, embs, pend, caches = [], [], [], []
    for sp in specs:
        vis, prompt, tok, emb, pending = prefix_rows(desc, seed, sp)
        toks.append(tok), embs.append(emb), pend.append(pending)
    eng.prefill(list(range(len(specs))), toks, embs)
    torch.cuda.synchronize()
    for i, (tok, emb) in enumerate(zip(toks, embs)):
        c = EngineCache(eng, desc, i)
        c.look()
        rows = np.where(tok[:, None] < 0, emb, O.embed_tokens(weights, np.maximum(tok, 0)))
        if len(rows):
            O.decoder_forward(desc, weights, rows.astype(np.float64), c, want_logits=False)
        caches.append(c)
    return pend, caches


@pytest.mark.parametrize("mode", ["region", "page"])
@pytest.mark.parametrize("dtype,maxb", [("fp32", 14), ("fp32", 300), ("bf16", 14), ("bf16", 300)])
def test_rounds_on_an_8bit_cache(dtype, mode, maxb):
    """Prefill, then rounds of verification and commit with accepted, cut and rejected drafts, blocks of one row among them; tables
    of 300 blocks have the keys split over workgroups."""
    desc, seed = MODELS[dtype], 31
    weights = W.make_weights(desc, seed)
    specs = [SequenceSpec(i, nv, npr, 0, 0.0) for i, (nv, npr) in enumerate([(40, 3), (5, 2), (110, 5), (16, 1), (0, 4), (33, 0)])]
    eng = make_engine(desc, weights, len(specs), maxb, 320)
    pend, caches = prefill(eng, desc, weights, seed, specs)
    rng = np.random.default_rng(5)
    for k in ([3, 0, 17, 64, 33, 1], [0, 0, 0, 0, 0, 0], [15, 1, 2, 5, 0, 9]):
        start = [len(c) for c in caches]
        blocks = [np.concatenate([[p], rng.integers(0, desc.vocab, n)]).astype(np.int32) for p, n in zip(pend, k)]
        out = eng.verify(list(range(len(specs))), blocks, mode, dump_rows=np.arange(sum(map(len, blocks))))
        alpha, bonus, status = eng.read_acceptance(len(specs))
        assert status == 0
        logits, argmax = out.logits.cpu().numpy(), out.argmax.cpu().numpy()
        force = np.array([min(n, f) for n, f in zip(k, (2, 0, 17, 30, 16, 0))], dtype=np.int32)   # rows kept of each draft
        for i, c in enumerate(caches):
            c.look()
            lo, hi = out.cu_q[i], out.cu_q[i + 1]
            a, b, u, ref = O.verify_block(desc, weights, c, pend[i], blocks[i][1:])
            err = float(np.abs(logits[lo:hi] - ref).max())
            assert err <= TOL[dtype], (i, err)
            margin = O.top2_margin(ref)
            assert len(gated_compare_argmax(argmax[lo:hi], u, margin)[0]) == 0
            if (margin > MARGIN_GATE).all():
                assert (alpha[i], bonus[i]) == (a, b)
            pend[i] = int(bonus[i])
            c.truncate(start[i] + 1 + force[i])
        eng.override_acceptance(force, bonus)
        eng.commit()
        torch.cuda.synchronize()
        assert eng.seq_len.cpu().tolist()[:len(specs)] == [len(c) for c in caches]
    eng.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_8bit_pass_touches_its_own_pages(dtype):
    """Pages of other sequences and full pages of earlier tokens keep their codes and scales."""
    desc, seed = MODELS[dtype], 32
    weights = W.make_weights(desc, seed)
    specs = [SequenceSpec(i, nv, 2, 0, 0.0) for i, nv in enumerate([20, 35, 7])]
    eng = make_engine(desc, weights, 3, 8, 64)
    pend, _ = prefill(eng, desc, weights, seed, specs)
    before = [t.clone() for t in (eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale)]
    eng.verify([1], [np.asarray([pend[1], 5, 6, 7, 8], dtype=np.int32)])
    torch.cuda.synchronize()
    table = eng.block_table.cpu().numpy()
    base = 36   # 35 visual rows and the prompt without its last token
    mine = set(table[1][base // 16:(base + 5 + 15) // 16].tolist())
    L, H = desc.n_layers, desc.n_kv_heads
    for t, (old, new) in enumerate(zip(before, (eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale))):
        differs = (old.view(L, eng.n_blocks, H, -1) != new.view(L, eng.n_blocks, H, -1)).any(-1).any(2).any(0).cpu().numpy()
        assert set(np.nonzero(differs)[0].tolist()) <= mine
    eng.close()


def test_greedy_decoding_is_verification_of_one_row():
    desc, seed = MODELS["bf16"], 33
    weights = W.make_weights(desc, seed)
    specs = [SequenceSpec(i, nv, 2, 0, 0.0) for i, nv in enumerate([20, 35])]
    eng = make_engine(desc, weights, 2, 8, 64)
    pend, _ = prefill(eng, desc, weights, seed, specs)
    eng.snapshot()
    codes = eng.k_pool.clone(), eng.v_pool.clone(), eng.k_scale.clone(), eng.v_scale.clone()
    got = eng.greedy_decode([0, 1], pend, 6)
    eng.restore()
    for t, c in zip((eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale), codes):
        t.copy_(c)
    tok = list(pend)
    for step in range(6):
        eng.verify([0, 1], [np.asarray([t], dtype=np.int32) for t in tok])
        _, bonus, status = eng.read_acceptance(2)
        assert status == 0 and bonus.tolist() == got[:, step].tolist()
        eng.commit()
        tok = bonus.tolist()
    eng.close()


def test_scores_of_a_verified_block():
    """Engine.score on a pass's logits; each log probability within 8 fp32 roundings of its magnitude and the sum's."""
    desc, seed = MODELS["bf16"], 34
    weights = W.make_weights(desc, seed)
    eng = make_engine(desc, weights, 1, 8, 64)
    pend, _ = prefill(eng, desc, weights, seed, [SequenceSpec(0, 20, 2, 0, 0.0)])
    block = np.asarray([pend[0], 9, 4, 7], dtype=np.int32)
    out = eng.verify([0], [block], dump_rows=np.arange(3))
    got = eng.score(out, block[1:], 3)
    x = out.logits.cpu().numpy().astype(np.float64)
    lse = np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)) + x.max(1)
    ref = x[np.arange(3), block[1:]] - lse
    tol = 2.0 ** -24 * (8 * (np.abs(x).max() + np.abs(lse)) + 32)
    assert (np.abs(got.logprob.cpu().numpy() - ref) <= tol).all()
    assert got.top_ids[:, 0].tolist() == out.argmax[:3].tolist()
    with pytest.raises(ValueError):
        eng.score(out, block)
    with pytest.raises(ValueError):
        eng.score(eng.verify([0], [block]), block)
    eng.close()


def test_passes_that_an_8bit_cache_refuses():
    """Everything here is refused on the host, before a launch."""
    from paper_2602_12957_amd.runtime import Engine, _ptr
    desc, seed = MODELS["bf16"], 35
    weights = W.make_weights(desc, seed)
    with pytest.raises(ValueError):
        Engine(desc, weights, 8, 1, 8, 32, kv_cache="int4")
    eng = make_engine(desc, weights, 2, 8, 64)
    block = np.asarray([1, 2, 3], dtype=np.int32)
    with pytest.raises(ValueError):
        eng.verify([0], [block], trees=[(np.asarray([3, 2, 3]), np.asarray([0, 1, 1]))])
    with pytest.raises(ValueError):
        eng.verify([0], [block], noalloc=True)
    b = eng.prepare([0], [block])
    ws = _ptr(eng.ws)

    def refused(code, layers=None, pool=None, w=ws, n=eng.ws_bytes, ctx=eng.ctx):
        for fn in (B.lib.hsd_verify_quant, B.lib.hsd_prefill_quant):
            assert fn(ctx, eng.stream, B.C.byref(pool or eng.cpool), eng.layers8 if layers is None else layers, B.C.byref(b), w, n) == code
    def changed(**kw):
        a = (B.hsd_kv_quant * desc.n_layers)(*eng.layers8)
        for k, v in kw.items():
            setattr(a[desc.n_layers - 1], k, v)
        return a
    refused(B.HSD_EINVAL, ctx=None)
    refused(B.HSD_EINVAL, w=None)
    refused(B.HSD_EINVAL, w=B.C.c_void_p(eng.ws.data_ptr() + 128))
    refused(B.HSD_ENOSPC, n=B.hsd_workspace_quant_bytes(eng.cdesc, 3, 1, 8) - 1)
    refused(B.HSD_EINVAL, layers=changed(n_blocks=eng.n_blocks - 1))
    refused(B.HSD_EINVAL, layers=changed(n_kv_heads=1))
    refused(B.HSD_EINVAL, layers=changed(k_scale=None))
    refused(B.HSD_EINVAL, pool=B.hsd_kv_pool(None, None, eng.n_blocks, None, _ptr(eng.free_count)))
    eng.close()


@pytest.mark.parametrize("dtype,maxb", [("fp32", 8), ("bf16", 300)])
def test_a_captured_8bit_pass_replays(dtype, maxb):
    """A pass and its commit in a graph, replayed with the engine's own passes between: the bits of the eager pass each time."""
    desc, seed = MODELS[dtype], 36
    weights = W.make_weights(desc, seed)
    eng = make_engine(desc, weights, 2, maxb, 64, n_blocks=16)
    specs = [SequenceSpec(i, nv, 2, 0, 0.0) for i, nv in enumerate([20, 35])]
    pend, _ = prefill(eng, desc, weights, seed, specs)
    b = eng.prepare([0, 1], [np.asarray([pend[0], 5, 6], dtype=np.int32), np.asarray([pend[1]], dtype=np.int32)])
    pages = (eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale)

    def step():
        eng.verify_prepared(b)
        eng.commit()

    def state():
        torch.cuda.synchronize()
        return [t.clone() for t in (eng.argmax[:4], eng.margin[:4], eng.accept_len[:2], eng.bonus[:2], eng.seq_len, eng.block_table) + pages]
    eng.snapshot()
    start = [t.clone() for t in pages]
    step()
    want = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        eng.restore()
        for t, s in zip(pages, start):
            t.copy_(s)
        graph.replay()
        for got, ref in zip(state(), want):
            assert torch.equal(got, ref)
        step()      # and a pass of the engine's own, further on
        torch.cuda.synchronize()
    assert int(eng.status.item()) == 0
    eng.close()


def test_rounds_with_the_plain_projections(monkeypatch):
    """HSD_DEBUG_FORCE_SIMPLE: other kernels in front of the same cache."""
    import functools
    import sys
    monkeypatch.setattr(sys.modules[__name__], "make_engine", functools.partial(make_engine, debug={"force_simple": 1}))
    test_rounds_on_an_8bit_cache("bf16", "region", 14)
