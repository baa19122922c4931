"""Calls around the 8-bit cache that come in other shapes than a packed batch that fits: rows behind the last sequence, more rows than
one workgroup places, rows of a block with gaps."""
import numpy as np
import pytest
import torch

from test_gpu_kvquant import HD, PAGE, RefCache, check_attend, cu_of, dev, fill, held, make_cache, rand_rows, ref_reserve

pytestmark = pytest.mark.gpu


def padded_step(cache, cu, k, v, q, out):
    n = k.shape[0]
    slots, pos = cache.reserve(cu, n)
    cache.append(k, v, slots)
    cache.attend(q, cu, out=out)
    return slots, pos


@pytest.mark.parametrize("total", [40, 600, 20000])
def test_rows_behind_the_last_sequence(total):
    """A captured step for `total` rows, replayed for batches that have fewer: their rows as in a batch of their own, the others and
    the pages of other sequences untouched."""
    rng = np.random.default_rng(total)
    maxb = total // PAGE + 10
    cache = make_cache(3 * maxb, 2, 3, maxb, shuffle=1)
    fill(cache, rng, [33, 7, 50], [0, 0, 0], torch.bfloat16)
    cache.snapshot()
    k, v = (rand_rows(rng, total, 2, torch.bfloat16).cuda() for _ in range(2))
    q, out = rand_rows(rng, total, 8, torch.bfloat16, 0.3).cuda(), torch.empty(total, 8, HD, dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    lens = [[5, 0, 20], [1, 1, 1], [0, 0, total - 3], [total // 2, 0, 0], [total - 2, 1, 1]]
    cu.copy_(cu_of(lens[0]))
    padded_step(cache, cu, k, v, q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots, pos = padded_step(cache, cu, k, v, q, out)
    for want in lens:
        n = sum(want)
        cache.restore()
        cu.copy_(cu_of(want))
        out.fill_(7.0)
        pages = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (slots, pos, out, cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
        assert bool((got[0][n:] == -1).all()) and bool((got[1][n:] == 0).all()) and bool((got[2][n:] == 7.0).all())
        cache.restore()
        for t, old in zip((cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale), pages):
            t.copy_(old)
        alone = torch.empty(n, 8, HD, dtype=torch.bfloat16, device="cuda")
        s, p = padded_step(cache, cu, k[:n], v[:n], q[:n], alone)
        assert torch.equal(got[0][:n], s) and torch.equal(got[1][:n], p) and int(cache.status.item()) == 0
        for t, g in zip((cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale), got[3:]):
            assert torch.equal(t, g)
        rows = {0, n - 1, n // 2} | set(rng.integers(0, n, 4).tolist())
        check_attend(cache, got[2][:n], q[:n], [33, 7, 50], want, torch.bfloat16, rows=rows)


@pytest.mark.parametrize("seed,n_seq,ctx_hi,q_hi", [(0, 1, 300, 17000), (1, 5, 100, 9000), (2, 3, 3000, 20000), (3, 700, 60, 60), (4, 4096, 40, 12)])
def test_more_rows_than_one_workgroup_places(seed, n_seq, ctx_hi, q_hi):
    """Above 16384 rows a second kernel writes places and positions."""
    rng = np.random.default_rng(seed)
    n_slots = n_seq + 2
    ctx, q = rng.integers(0, ctx_hi + 1, n_slots), rng.integers(q_hi * 2 // 3, q_hi + 1, n_seq)
    q[rng.random(n_seq) < 0.1] = 0
    q[0] = max(q[0], 17000 if n_seq < 100 else 0)
    slots = rng.permutation(n_slots)[:n_seq]
    maxb = int((ctx_hi + q.max()) // PAGE + 1) - (seed == 2)     # (one table that is too short)
    n_blocks = int((ctx // PAGE + 1).sum() + (q // PAGE + 2).sum())
    cache = make_cache(n_blocks, 1, n_slots, maxb, shuffle=seed)
    ids = cache.free_list.cpu().numpy()
    table, at = np.full((n_slots, maxb), -1, np.int32), 0
    for i, c in enumerate(ctx):
        b = -(-int(c) // PAGE)
        table[i, :b] = ids[n_blocks - at - b:n_blocks - at][::-1]
        at += b
    cache.block_table.copy_(dev(table)), cache.seq_len.copy_(dev(ctx.astype(np.int32))), cache.free_count.fill_(n_blocks - at)
    if seed == 2:
        ctx[slots[0]] = maxb * PAGE - int(q[0]) + 20
        cache.seq_len.copy_(dev(ctx.astype(np.int32)))
    want = ref_reserve(ids, n_blocks - at, table, ctx, q, slots, n_blocks)
    total = int(q.sum())
    assert total > 16384
    row_slot, row_pos = cache.reserve(cu_of(q), total, dev(slots.astype(np.int32)))
    np.testing.assert_array_equal(row_slot.cpu().numpy(), want[0])
    np.testing.assert_array_equal(row_pos.cpu().numpy(), want[1])
    np.testing.assert_array_equal(cache.block_table.cpu().numpy(), want[2])
    assert int(cache.free_count.item()) == want[3] and int(cache.status.item()) == want[4] == (2 if seed == 2 else 0)


class GappedCache(RefCache):
    """The plain cache, for rows of a block that leave slots out: those before the last row keep their values."""

    def append(self, k, v, slots):
        runs = {}
        for r, sl in enumerate(slots):
            runs.setdefault(int(sl) // PAGE, []).append((int(sl) % PAGE, r))
        for b, rows in runs.items():
            for i, src in enumerate((k, v)):
                page = self.x[i, b].copy()
                page[:, rows[-1][0] + 1:] = 0.0
                for off, r in rows:
                    page[:, off] = src[r]
                for h in range(page.shape[0]):
                    self.x[i, b, h], self.e[i, b, h] = held(page[h])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,n_blocks", [(1, 3), (2, 40), (3, 1500)])
def test_rows_of_a_block_with_gaps(dtype, heads, n_blocks):
    """Rows in the order of their slots that leave some out, block after block in any order; few rows (one a wave) and many (16)."""
    rng = np.random.default_rng(heads)
    cache, ref = make_cache(n_blocks, heads, 1, n_blocks), GappedCache(n_blocks, heads)
    for keep in (1.0, 0.6, 0.2, 0.9):
        slots = np.concatenate([b * PAGE + np.nonzero(rng.random(PAGE) < keep)[0] for b in rng.permutation(n_blocks)]).astype(np.int32)
        k, v = rand_rows(rng, len(slots), heads, dtype), rand_rows(rng, len(slots), heads, dtype) * 11.0
        k[::7] *= 50.0
        cache.append(k.cuda(), v.cuda(), dev(slots))
        ref.append(k.double().numpy(), v.double().numpy(), slots)
        every = np.arange(n_blocks * PAGE, dtype=np.int32)
        got = cache.read(dev(every), torch.float32)
        for g, x in zip(got, ref.x):
            np.testing.assert_array_equal(g.double().cpu().numpy(), x[every // PAGE, :, every % PAGE])
    assert int(cache.status.item()) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,lens,heads,maxb", [([300, 20], [60, 1], (8, 2), None), ([5000, 9], [1, 3], (16, 4), 400), ([50], [2100], (64, 64), None)])
def test_output_in_place_of_the_queries(dtype, ctx, lens, heads, maxb):
    rng = np.random.default_rng(4)
    need = max(-(-(c + n) // PAGE) for c, n in zip(ctx, lens))
    cache = make_cache(len(ctx) * need, heads[1], len(ctx), maxb or need, shuffle=1)
    fill(cache, rng, ctx, lens, dtype)
    q, cu = rand_rows(rng, sum(lens), heads[0], dtype, 0.3).cuda(), cu_of(lens)
    want = cache.attend(q, cu)
    assert cache.attend(q, cu, out=q) is q and torch.equal(q, want)
