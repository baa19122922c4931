"""Decoder passes on an 8-bit cache at sizes and with rules that the rounds against the oracle do not reach: passes whose rows are appended
16 a wave and attend 64 columns a wave, and the relaxed acceptance rule."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from workloads.generators import SequenceSpec

from hsd_testlib import MARGIN_GATE
from test_gpu_kvquant_decoder import MODELS, TOL, held_pages, make_engine, prefill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows", [("bf16", 4264), ("fp32", 8208)])
def test_one_large_prefill_is_many_small_ones(dtype, rows):
    """Keys and values of the first layer do not depend on attention: the same codes and scales, bit by bit, whether four sequences come in
    one pass or in passes of 16 blocks each.  Further layers differ by rounding: by a step of their codes (2^-3 of the value) where that falls on
    the other side of a border, beyond the bar of a pass."""
    desc = MODELS[dtype]
    weights = W.make_weights(desc, 41)
    rng = np.random.default_rng(41)
    toks = [rng.integers(0, desc.vocab, rows - 16 * i).astype(np.int32) for i in range(4)]
    maxb, held, raw = rows // 16 + 1, [], []
    for chunk in (4 * rows, 4 * 256):
        eng = make_engine(desc, weights, 4, maxb, 4 * rows, n_blocks=4 * maxb, max_dump=1)
        eng.prefill(range(4), toks, chunk=chunk)
        torch.cuda.synchronize()
        assert int(eng.status.item()) == 0 and eng.seq_len.tolist() == [len(t) for t in toks]
        table = eng.block_table.cpu().numpy()
        ids = np.concatenate([table[i, :-(-len(t) // 16)] for i, t in enumerate(toks)])
        L, per = desc.n_layers, desc.n_kv_heads * 1024
        raw.append([t.cpu().numpy().reshape(L, -1, w)[0, ids] for t, w in ((eng.k_pool, per), (eng.v_pool, per), (eng.k_scale, desc.n_kv_heads),
                                                                           (eng.v_scale, desc.n_kv_heads))])
        k, v, s = held_pages(eng, desc)
        held.append((k[:, ids], v[:, ids], s[:, :, ids]))
        eng.close()
    for a, b in zip(*raw):
        np.testing.assert_array_equal(a, b)
    scale = np.maximum(held[0][2], held[1][2])
    for i in range(2):
        for layer in range(1, desc.n_layers):
            a, b = held[0][i][layer], held[1][i][layer]
            bar = TOL[dtype] * max(1.0, np.abs(b).max())
            tol = bar + 2.0 ** -3 * (np.abs(b) + bar) + 2.0 ** -9 * scale[i, layer][:, :, None, None]
            assert (np.abs(a - b) <= tol).all(), (i, layer, float((np.abs(a - b) / tol).max()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [0.75, 0.3])
def test_relaxed_acceptance_on_an_8bit_cache(dtype, tau):
    """alpha, bonus and gaps are what the rule gives on the pass's own logits (no deciding gap lies at the threshold)."""
    desc, seed, lt = MODELS[dtype], 42, math.log(tau)
    weights = W.make_weights(desc, seed)
    specs = [SequenceSpec(i, nv, npr, 0, 0.0) for i, (nv, npr) in enumerate([(40, 3), (5, 2), (100, 5), (16, 1)])]
    eng = make_engine(desc, weights, len(specs), 16, 320)
    pend, _ = prefill(eng, desc, weights, seed, specs)
    rng = np.random.default_rng(7)
    eng.snapshot()
    pages = [t.clone() for t in (eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale)]
    drafts = [rng.integers(0, desc.vocab, n).astype(np.int32) for n in (30, 0, 64, 7)]
    accepted = 0
    for turn in range(12):     # drafts that follow the model's first or second choice ever further
        eng.restore()
        for t, old in zip((eng.k_pool, eng.v_pool, eng.k_scale, eng.v_scale), pages):
            t.copy_(old)
        blocks = [np.concatenate([[p], d]).astype(np.int32) for p, d in zip(pend, drafts)]
        out = eng.verify(range(len(specs)), blocks, dump_rows=np.arange(sum(map(len, blocks))), log_tau=lt)
        alpha, bonus, status = eng.read_acceptance(len(specs))
        assert status == 0
        logits, gap = out.logits.cpu().numpy(), out.gap.cpu().numpy()
        for i, d in enumerate(drafts):
            x = logits[out.cu_q[i]:out.cu_q[i + 1]]
            want = np.array([x[r, t] - x[r].max() for r, t in enumerate(d)])
            np.testing.assert_allclose(gap[out.cu_q[i] + 1:out.cu_q[i + 1]], want, rtol=0, atol=1e-5)
            if len(d) and np.abs(want - lt).min() < MARGIN_GATE:
                continue
            a = int(np.argmin(np.append(want >= lt, False)))
            assert alpha[i] == a and bonus[i] == x[a].argmax()
            accepted += a
            order = np.argsort(-x, axis=1)
            drafts[i] = d.copy()
            drafts[i][a:a + 1] = order[a, rng.integers(0, 2)] if a < len(d) else []
    assert accepted > 0
    eng.close()
