"""The 8-bit cache on the GPU against plain implementations in 64 bits: placing rows, appending, reading, attending."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE, HD = 16, 64
EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


# ---------------------------------------------------------------------------------------------------- references
def ref_reserve(free_list, free_count, table, seq_len, q, slots, n_blocks):
    """Returns (row_slot, row_pos, table, free_count, status); the free list itself is only read."""
    table, need, status = table.copy(), [], 0
    for s, n in enumerate(q):
        sl = slots[s]
        hi = -(-(seq_len[sl] + n) // PAGE) if n else 0
        if hi > table.shape[1]:
            status, hi = status | 2, table.shape[1]
        need += [(sl, i) for i in range(seq_len[sl] // PAGE, hi) if table[sl, i] < 0]
    if len(need) > free_count:
        status |= 1
    else:
        for j, (sl, i) in enumerate(need):
            table[sl, i] = free_list[free_count - 1 - j]
        free_count -= len(need)
    row_slot, row_pos = [], []
    for s, n in enumerate(q):
        for r in range(n):
            pos = seq_len[slots[s]] + r
            b = table[slots[s], pos // PAGE] if pos // PAGE < table.shape[1] else -1
            row_slot.append(b * PAGE + pos % PAGE if 0 <= b < n_blocks else -1)
            row_pos.append(pos)
    return np.array(row_slot, np.int32), np.array(row_pos, np.int32), table, free_count, status


def e4m3(y):
    """Nearest e4m3 value, ties to even, of |y| <= 448 (fp64)."""
    e = np.maximum(np.frexp(y)[1] - 1, -6) - 3
    return np.ldexp(np.rint(np.ldexp(y, -e)), e)


def held(page):
    """What a page [16, 64] of finite values holds: (values, exponent)."""
    top = np.abs(page).max()
    e = 0
    if top > 0:
        e = -100
        while e < 119 and math.ldexp(448.0, e) < top:
            e += 1
    lim = math.ldexp(448.0, 119)
    return np.ldexp(e4m3(np.ldexp(np.clip(page, -lim, lim), -e)), e), e


class RefCache:
    """value[block][head][token][dim] in fp64, written page by page as the cache is."""

    def __init__(self, n_blocks, heads):
        self.x = np.zeros((2, n_blocks, heads, PAGE, HD))
        self.e = np.zeros((2, n_blocks, heads), np.int64)

    def append(self, k, v, slots):
        lim = math.ldexp(448.0, 119)
        runs = {}
        for r, sl in enumerate(slots):
            if sl >= 0:
                runs.setdefault(int(sl) // PAGE, []).append((int(sl) % PAGE, r))
        for b, rows in runs.items():
            for i, src in enumerate((k, v)):
                page = self.x[i, b].copy()
                page[:, rows[0][0]:] = 0.0
                for off, r in rows:
                    page[:, off] = np.clip(np.nan_to_num(src[r], nan=0.0, posinf=lim, neginf=-lim), -lim, lim)
                for h in range(page.shape[0]):
                    self.x[i, b, h], self.e[i, b, h] = held(page[h])


def bound_attend(q, keys, vals, scale, visible, dtype):
    """(reference, tolerance) of one row and head: softmax(scale q.k) v over the visible keys.

    Rounding counted: the output (half a step); the probabilities of a bf16 call (half a step each, numerator and
    denominator alike, so that o moves by at most half a step of sum p |v - o|); fp32 products and sums of 64 terms in a score (68
    roundings of the sum of magnitudes), the exponential (argument and result, 8 roundings of its magnitude), sums over
    keys (one rounding a key and three for the parts and their factors)."""
    kk, vv = keys[visible], vals[visible]
    if len(kk) == 0:
        return np.zeros(HD), np.zeros(HD)
    s = kk @ q * scale
    p = np.exp(s - s.max())
    p /= p.sum()
    o = p @ vv
    u = 2.0 ** -24
    mags = np.abs(kk) @ np.abs(q) * abs(scale)
    ds = u * (68 * mags.max() + 8 * (np.abs(s).max() + 40))
    spread = p @ np.abs(vv - o)
    tol = EPS[dtype] * np.abs(o) + 2 * ds * spread + (len(kk) + 8) * u * (p @ np.abs(vv)) + 1e-37
    if dtype == torch.bfloat16:
        tol = tol + EPS[dtype] * spread
    return o, 1.01 * tol


# ---------------------------------------------------------------------------------------------------- helpers
def make_cache(n_blocks, heads, n_slots, maxb, layers=1, shuffle=None):
    from paper_2602_12957_amd.kvquant import QuantKV
    c = QuantKV(n_blocks, heads, n_slots, maxb, n_layers=layers)
    if shuffle is not None:
        c.free_list.copy_(torch.from_numpy(np.random.default_rng(shuffle).permutation(n_blocks).astype(np.int32)))
    return c


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def cu_of(q):
    return dev(np.concatenate([[0], np.cumsum(q)]).astype(np.int32))


def rand_rows(rng, n, heads, dtype, spread=0.7):
    x = rng.standard_normal((n, heads, HD)) * np.exp(spread * rng.standard_normal((heads, HD)))
    return torch.from_numpy(x).to(dtype)


def fill(cache, rng, ctx, q, dtype, slots=None, k_mul=1.0):
    """ctx tokens, then the q rows of every sequence; seq_len stays ctx.  Returns nothing: read the cache for its values."""
    slot_t = None if slots is None else dev(np.array(slots, np.int32))
    for lens, keep in ((ctx, True), (q, False)):
        if sum(lens) == 0:
            continue
        cu, n = cu_of(lens), int(sum(lens))
        row_slot, _ = cache.reserve(cu, n, slot_t)
        for l in range(cache.n_layers):
            k, v = rand_rows(rng, n, cache.n_kv_heads, dtype), rand_rows(rng, n, cache.n_kv_heads, dtype)
            cache.append((k * k_mul).cuda(), v.cuda(), row_slot, layer=l)
        if keep:
            cache.commit(cu, n, seq_slot=slot_t)
    assert int(cache.status.item()) == 0


def sequence_values(cache, slot, n, layer=0):
    """(keys, values) [n, heads, 64] in fp64 as the cache holds them"""
    if n == 0:
        return np.zeros((2, 0, cache.n_kv_heads, HD))
    table = cache.block_table[slot].cpu().numpy()
    pos = np.arange(n)
    k, v = cache.read(dev((table[pos // PAGE] * PAGE + pos % PAGE).astype(np.int32)), torch.float32, layer)
    return np.stack([k.cpu().numpy(), v.cpu().numpy()]).astype(np.float64)


def check_attend(cache, out, q, ctx, lens, dtype, scale=0.125, slots=None, layer=0, rows=None, hidden=None):
    """Every row (or the given ones) against the bound; hidden: positions per sequence that have no valid block."""
    out, q = out.float().cpu().numpy().astype(np.float64), q.float().cpu().numpy().astype(np.float64)
    group = q.shape[1] // cache.n_kv_heads
    base, worst = 0, 0.0
    for s, (c, n) in enumerate(zip(ctx, lens)):
        kv = sequence_values(cache, s if slots is None else slots[s], c + n, layer)
        for i in range(n):
            if rows is not None and base + i not in rows:
                continue
            visible = np.arange(c + n) <= c + i
            if hidden is not None:
                visible &= ~np.isin(np.arange(c + n), hidden[s])
            for h in range(q.shape[1]):
                ref, tol = bound_attend(q[base + i, h], kv[0][:, h // group], kv[1][:, h // group], scale, visible, dtype)
                err = np.abs(out[base + i, h] - ref)
                assert np.isfinite(err).all() and (err <= tol).all(), (s, i, h, float((err / np.maximum(tol, 1e-300)).max()))
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
        base += n
    return worst


# ---------------------------------------------------------------------------------------------------- placing
@pytest.mark.parametrize("seed,n_seq,ctx_hi,q_hi", [(0, 1, 40, 1), (1, 5, 100, 3), (2, 64, 300, 70), (3, 700, 60, 40), (4, 3, 2000, 3000), (5, 4096, 50, 3)])
def test_reserve_and_commit_against_the_definition(seed, n_seq, ctx_hi, q_hi):
    rng = np.random.default_rng(seed)
    n_slots = n_seq + 3
    ctx, q = rng.integers(0, ctx_hi + 1, n_slots), rng.integers(0, q_hi + 1, n_seq)
    q[0] = max(q[0], 1)
    slots = rng.permutation(n_slots)[:n_seq]
    maxb = int((ctx_hi + q_hi) // PAGE + 2)
    n_blocks = int((ctx // PAGE + 1).sum() + (q // PAGE + 2).sum())
    cache = make_cache(n_blocks, 1, n_slots, maxb, shuffle=seed)
    # what is cached already sits in random blocks
    have = [-(-int(c) // PAGE) for c in ctx]
    ids = cache.free_list.cpu().numpy()
    table, at = np.full((n_slots, maxb), -1, np.int32), 0
    for i, b in enumerate(have):
        table[i, :b] = ids[n_blocks - at - b:n_blocks - at][::-1]
        at += b
    cache.block_table.copy_(dev(table)), cache.seq_len.copy_(dev(ctx.astype(np.int32))), cache.free_count.fill_(n_blocks - at)
    want = ref_reserve(ids, n_blocks - at, table, ctx, q, slots, n_blocks)
    cu, total, st = cu_of(q), int(q.sum()), dev(slots.astype(np.int32))
    row_slot, row_pos = cache.reserve(cu, total, st)
    np.testing.assert_array_equal(row_slot.cpu().numpy(), want[0])
    np.testing.assert_array_equal(row_pos.cpu().numpy(), want[1])
    np.testing.assert_array_equal(cache.block_table.cpu().numpy(), want[2])
    assert int(cache.free_count.item()) == want[3] and int(cache.status.item()) == want[4] == 0
    # a second reservation for the same rows finds the blocks there
    again, _ = cache.reserve(cu, total, st)
    np.testing.assert_array_equal(again.cpu().numpy(), want[0])
    assert int(cache.free_count.item()) == want[3]
    # part of the rows accepted, some sequences rolled back: blocks beyond return, none is lost
    accept = rng.integers(-1, q_hi + 1, n_seq).astype(np.int32)
    cache.commit(cu, total, dev(accept), st)
    new_len = ctx.copy()
    for s in range(n_seq):
        a = min(int(accept[s]), int(q[s]) - 1)
        if a >= 0:
            new_len[slots[s]] += 1 + a
    np.testing.assert_array_equal(cache.seq_len.cpu().numpy(), new_len)
    table = cache.block_table.cpu().numpy()
    for i in range(n_slots):
        keep = -(-int(new_len[i]) // PAGE)
        np.testing.assert_array_equal(table[i, :keep], want[2][i, :keep])
        if i in slots:
            assert (table[i, keep:] == -1).all()
    held_ids = np.concatenate([table[table >= 0], cache.free_list.cpu().numpy()[:int(cache.free_count.item())]])
    np.testing.assert_array_equal(np.sort(held_ids), np.arange(n_blocks))


def test_reserve_reports_a_short_pool_a_short_table_and_a_bad_slot():
    cache = make_cache(6, 1, 2, 4)
    cu = cu_of([30, 70])
    row_slot, row_pos = cache.reserve(cu, 100)       # 2 + 5 blocks, but a table of 4 entries: 6 in all
    assert int(cache.status.item()) == 2
    slot = row_slot.cpu().numpy()
    assert (slot[:94] >= 0).all() and (slot[94:] == -1).all() and int(cache.free_count.item()) == 0
    np.testing.assert_array_equal(row_pos.cpu().numpy(), np.concatenate([np.arange(30), np.arange(70)]))
    cache.reset()
    cache.free_count.fill_(3)
    row_slot, _ = cache.reserve(cu_of([30, 33]), 63)  # 5 blocks of 3: nothing is taken
    assert int(cache.status.item()) == 1 and int(cache.free_count.item()) == 3
    assert (row_slot.cpu().numpy() == -1).all() and (cache.block_table.cpu().numpy() == -1).all()
    cache.reset()
    cache.reserve(cu_of([3]), 3, dev(np.array([7], np.int32)))
    assert int(cache.status.item()) == 4


def test_reserve_of_no_rows():
    cache = make_cache(6, 1, 2, 4)
    a, b = cache.reserve(cu_of([0, 0]), 0)
    assert a.numel() == b.numel() == 0 and int(cache.free_count.item()) == 6 and int(cache.status.item()) == 0
    cache.commit(cu_of([0, 0]), 0)
    assert int(cache.seq_len.sum().item()) == 0


# ---------------------------------------------------------------------------------------------------- appending, reading
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,steps", [(1, [[1]]), (2, [[5, 0, 40], [1, 1, 1], [20, 33, 2], [1, 0, 1]]), (3, [[15, 16, 17], [1, 1, 1], [1, 1, 1]]),
                                         (4, [[700, 300], [1, 500]]), (2, [[1500, 3000], [2600, 1]])])
def test_append_and_read_against_the_definition(dtype, heads, steps):
    rng = np.random.default_rng(len(steps) * 7 + heads)
    n_seq = len(steps[0])
    total = sum(sum(s) for s in steps)
    n_blocks = total // PAGE + 2 * n_seq + 1
    cache = make_cache(n_blocks, heads, n_seq, total // PAGE + 2, shuffle=3)
    ref = RefCache(n_blocks, heads)
    for q in steps:
        n, cu = sum(q), cu_of(q)
        k, v = rand_rows(rng, n, heads, dtype), rand_rows(rng, n, heads, dtype) * 37.0
        k[0] *= 1000.0       # a token that moves its page's scale
        row_slot, _ = cache.reserve(cu, n)
        cache.append(k.cuda(), v.cuda(), row_slot)
        cache.commit(cu, n)
        slots = row_slot.cpu().numpy()
        ref.append(k.double().numpy(), v.double().numpy(), slots)
    every = np.array([b * PAGE + t for row in cache.block_table.cpu().numpy() for b in row if b >= 0 for t in range(PAGE)], np.int32)
    rng.shuffle(every)
    for t in (torch.float32, torch.bfloat16):
        gk, gv = cache.read(dev(every), t)
        np.testing.assert_array_equal(gk.double().cpu().numpy(), ref.x[0][every // PAGE, :, every % PAGE])
        np.testing.assert_array_equal(gv.double().cpu().numpy(), ref.x[1][every // PAGE, :, every % PAGE])
    used = np.unique(every // PAGE)
    np.testing.assert_array_equal(cache.k_scale[0].double().cpu().numpy()[used], 2.0 ** ref.e[0][used])
    np.testing.assert_array_equal(cache.v_scale[0].double().cpu().numpy()[used], 2.0 ** ref.e[1][used])
    assert int(cache.status.item()) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_extreme_values(dtype):
    """Zeros, the smallest and largest magnitudes, ties between codes, NaN and infinities; a page full of junk is overwritten."""
    cache = make_cache(8, 1, 1, 8)
    cache.k_codes.fill_(0x7f), cache.v_codes.fill_(0xff)
    cache.k_scale.fill_(math.nan), cache.v_scale.fill_(math.inf)
    fi = torch.finfo(dtype)
    codes = np.array([e4m3(np.float64(x)) for x in np.linspace(1, 2, 17)])
    rows = [np.zeros(HD), np.full(HD, fi.tiny), np.linspace(-448, 448, HD), np.linspace(0.5, 0.5625, HD), np.resize(codes, HD),
            np.full(HD, 448.0), np.full(HD, 449.0), np.ldexp(1.0, np.arange(HD) - 40), np.full(HD, -0.0)]
    big = [np.full(HD, fi.max), np.resize([fi.max, -1.0, 1e30, -fi.max], HD)]
    for group, bits in ((rows, 0), (rows[:1], 0), (big, 0), ([np.resize([np.nan, 2.0, np.inf, -np.inf, -3.0], HD)], 16), ([np.full(HD, np.nan)], 16)):
        cache.reset()
        ref = RefCache(8, 1)
        x = torch.from_numpy(np.stack(group))[:, None].to(dtype)
        row_slot, _ = cache.reserve(cu_of([len(group)]), len(group))
        cache.append(x.cuda(), (-x).cuda(), row_slot)
        ref.append(x.double().numpy(), -x.double().numpy(), row_slot.cpu().numpy())
        at = np.arange(PAGE) + int(row_slot[0].item()) // PAGE * PAGE
        gk, gv = cache.read(dev(at.astype(np.int32)), torch.float32)
        np.testing.assert_array_equal(gk.double().cpu().numpy(), ref.x[0][at // PAGE, :, at % PAGE])
        np.testing.assert_array_equal(gv.double().cpu().numpy(), ref.x[1][at // PAGE, :, at % PAGE])
        assert int(cache.status.item()) == bits


def test_append_takes_slices_of_wider_rows_and_leaves_unplaced_rows_out():
    rng = np.random.default_rng(5)
    heads, n = 2, 37
    wide = torch.from_numpy(rng.standard_normal((n, 777))).to(torch.bfloat16).cuda()
    k, v = wide[:, 3:3 + heads * HD].unflatten(1, (heads, HD)), wide[:, 401:401 + heads * HD].unflatten(1, (heads, HD))   # odd elements
    cache, ref = make_cache(9, heads, 1, 9), RefCache(9, heads)
    row_slot, _ = cache.reserve(cu_of([n]), n)
    row_slot[20:32] = torch.tensor([-1, -5, 9 * PAGE, 1 << 30] * 3, dtype=torch.int32)     # no place, or one beyond the pool
    cache.append(k, v, row_slot)
    keep = [r for r in range(n) if r < 20 or r >= 32]
    slots = row_slot.cpu().numpy()
    got_k, got_v = cache.read(row_slot)
    ref.append(k[keep].double().cpu().numpy(), v[keep].double().cpu().numpy(), slots[keep])
    np.testing.assert_array_equal(got_k[keep].double().cpu().numpy(), ref.x[0][slots[keep] // PAGE, :, slots[keep] % PAGE])
    np.testing.assert_array_equal(got_v[keep].double().cpu().numpy(), ref.x[1][slots[keep] // PAGE, :, slots[keep] % PAGE])
    assert (got_k[20:32] == 0).all() and (got_v[20:32] == 0).all()


def test_append_touches_its_own_pages_and_layer_alone():
    rng = np.random.default_rng(6)
    cache = make_cache(12, 2, 2, 6, layers=3)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_(torch.from_numpy(rng.integers(0, 256, t.shape).astype(np.uint8)))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.from_numpy(rng.random(t.shape).astype(np.float32)))
    before = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
    row_slot, _ = cache.reserve(cu_of([17, 3]), 20)
    k = rand_rows(rng, 20, 2, torch.bfloat16).cuda()
    cache.append(k, k, row_slot, layer=1)
    mine = torch.zeros((3, 12), dtype=torch.bool)
    mine[1, torch.unique(row_slot.cpu() // PAGE).long()] = True
    for t, old in zip((cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale), before):
        assert torch.equal(t[~mine.cuda()], old[~mine.cuda()])


# ---------------------------------------------------------------------------------------------------- attending
SHAPES = [  # ctx, rows, (query heads, kv heads)
    ([0], [1], (4, 4)), ([1055], [1], (16, 4)), ([0, 15, 16, 17, 300], [1, 1, 1, 1, 1], (8, 2)), ([5, 40, 100], [0, 1, 3], (5, 1)),
    ([31, 0, 64], [17, 33, 2], (6, 2)), ([100, 7], [65, 130], (16, 4)), ([513, 2], [40, 1], (16, 2)), ([200], [70], (12, 4)), ([64, 64], [16, 64], (32, 2)),
    ([9, 33], [25, 48], (2, 2)), ([70, 1], [3, 1], (40, 1))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,lens,heads", SHAPES)
def test_attend_against_the_definition(dtype, ctx, lens, heads):
    rng = np.random.default_rng(sum(ctx) + heads[0])
    n_seq, total = len(ctx), sum(lens)
    maxb = max((c + n) // PAGE + 1 for c, n in zip(ctx, lens)) + 2
    cache = make_cache(n_seq * maxb, heads[1], n_seq + 2, maxb, shuffle=1)
    cache.k_codes.fill_(0x7f), cache.v_codes.fill_(0x7f)      # NaN wherever nothing was appended
    slots = list(rng.permutation(n_seq + 2)[:n_seq])
    fill(cache, rng, ctx, lens, dtype, slots)
    q = rand_rows(rng, total, heads[0], dtype, 0.3).cuda()
    out = cache.attend(q, cu_of(lens), dev(np.array(slots, np.int32)))
    check_attend(cache, out, q, ctx, lens, dtype, slots=slots)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,lens,heads", [([9000, 4111, 130, 0], [1, 1, 1, 1], (8, 2)), ([5000, 2047], [5, 9], (4, 1)), ([1500, 3000], [300, 700], (8, 2)),
                                            ([700] * 12, [90] * 12, (16, 4)), ([40000], [1], (16, 4)), ([3100], [2100], (4, 4))])
def test_attend_of_long_caches_and_blocks(dtype, ctx, lens, heads):
    rng = np.random.default_rng(sum(ctx))
    n_seq, total = len(ctx), sum(lens)
    maxb = max((c + n) // PAGE + 1 for c, n in zip(ctx, lens))
    cache = make_cache(sum((c + n) // PAGE + 2 for c, n in zip(ctx, lens)), heads[1], n_seq, maxb, shuffle=2)
    fill(cache, rng, ctx, lens, dtype)
    q = rand_rows(rng, total, heads[0], dtype, 0.3).cuda()
    out = cache.attend(q, cu_of(lens))
    ends = np.cumsum(lens)
    rows = set(ends - 1) | set(ends - np.array(lens)) | set(rng.integers(0, total, 24).tolist())
    check_attend(cache, out, q, ctx, lens, dtype, rows=rows)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_with_scores_far_apart(dtype):
    """Scores of hundreds, falling and rising along the keys, and a scale that turns them round: the reference has to move."""
    rng = np.random.default_rng(9)
    for mul, scale in ((60.0, 0.125), (60.0, -0.125), (1.0, 0.0), (1e-20, 0.125), (1e18, 1e-19)):
        ctx, lens = [200, 40], [3, 50]
        cache = make_cache(40, 2, 2, 20)
        fill(cache, rng, ctx, lens, dtype, k_mul=mul)
        q = rand_rows(rng, 53, 4, dtype, 0.3).cuda()
        out = cache.attend(q, cu_of(lens), scale=scale)
        check_attend(cache, out, q, ctx, lens, dtype, scale=scale)


def test_attend_a_query_that_is_not_finite_leaves_the_others_alone():
    rng = np.random.default_rng(10)
    ctx, lens = [100], [40]
    cache = make_cache(12, 1, 1, 12)
    fill(cache, rng, ctx, lens, torch.bfloat16)
    q = rand_rows(rng, 40, 4, torch.bfloat16, 0.3).cuda()
    want = cache.attend(q, cu_of(lens))
    bad = q.clone()
    bad[7, 1, 5], bad[21, 0, 0], bad[30, 3] = math.nan, math.inf, 3e38
    got = cache.attend(bad, cu_of(lens))
    mine = torch.zeros(40, 4, dtype=torch.bool)
    mine[7, 1] = mine[21, 0] = mine[30, 3] = True
    assert torch.equal(got[~mine.cuda()], want[~mine.cuda()])
    assert torch.isnan(got[7, 1]).all() and torch.isnan(got[21, 0]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_leaves_out_positions_without_a_block(dtype):
    """Entries that are negative or beyond the pool hide their 16 positions; rows that see nothing become 0."""
    rng = np.random.default_rng(11)
    ctx, lens = [90, 0, 33], [20, 40, 1]
    cache = make_cache(30, 2, 3, 10)
    fill(cache, rng, ctx, lens, dtype)
    table = cache.block_table.clone()
    hidden = [list(range(16, 48)), list(range(0, 32)), list(range(0, 48))]
    q = rand_rows(rng, 61, 6, dtype, 0.3).cuda()
    kv = [sequence_values(cache, s, c + n) for s, (c, n) in enumerate(zip(ctx, lens))]
    cache.block_table[0, 1], cache.block_table[0, 2], cache.block_table[1, 0], cache.block_table[1, 1] = -1, 30, -7, 1 << 30
    cache.block_table[2, :] = -1
    out = cache.attend(q, cu_of(lens))
    cache.block_table.copy_(table)
    check_attend(cache, out, q, ctx, lens, dtype, hidden=hidden)
    assert (out[20:52] == 0).all() and (out[60] == 0).all()
    assert len(kv) == 3


def test_attend_of_slices_writes_its_rows_alone():
    """Queries as a slice of a fused projection at an odd element, output rows far apart: what lies between stays."""
    rng = np.random.default_rng(12)
    ctx, lens = [50, 3], [2, 40]
    cache = make_cache(12, 2, 2, 8)
    fill(cache, rng, ctx, lens, torch.bfloat16)
    wide = torch.from_numpy(rng.standard_normal((42, 1001))).to(torch.bfloat16).cuda()
    q = wide[:, 5:5 + 4 * HD].unflatten(1, (4, HD))
    frame = torch.full((44, 999), 7.0, dtype=torch.bfloat16, device="cuda")
    out = frame[:42, 1:1 + 4 * HD].unflatten(1, (4, HD))
    assert cache.attend(q, cu_of(lens), out=out) is out
    check_attend(cache, out, q, ctx, lens, torch.bfloat16)
    frame[:42, 1:1 + 4 * HD] = 7.0
    assert (frame == 7.0).all()


def test_a_token_by_token_run_of_all_calls():
    """Two sequences grow token by token through reserve, append, attend and commit, with a draft rolled back on the way."""
    rng = np.random.default_rng(13)
    cache = make_cache(20, 2, 2, 10, layers=2, shuffle=4)
    ref = [RefCache(20, 2), RefCache(20, 2)]
    lens = np.zeros(2, np.int64)
    for step in range(40):
        q = [1, 1] if step % 5 else [4, 7]
        n, cu = sum(q), cu_of(q)
        row_slot, row_pos = cache.reserve(cu, n)
        np.testing.assert_array_equal(row_pos.cpu().numpy(), np.concatenate([l + np.arange(m) for l, m in zip(lens, q)]))
        for l in range(2):
            k, v = rand_rows(rng, n, 2, torch.bfloat16), rand_rows(rng, n, 2, torch.bfloat16)
            cache.append(k.cuda(), v.cuda(), row_slot, layer=l)
            ref[l].append(k.double().numpy(), v.double().numpy(), row_slot.cpu().numpy())
            x = rand_rows(rng, n, 4, torch.bfloat16, 0.3).cuda()
            out = cache.attend(x, cu, layer=l)
            check_attend(cache, out, x, lens, q, torch.bfloat16, layer=l)
            table = cache.block_table.cpu().numpy()
            for s in range(2):
                pos = np.arange(lens[s] + q[s])
                at = table[s, pos // PAGE] * PAGE + pos % PAGE
                np.testing.assert_array_equal(sequence_values(cache, s, len(pos), l)[0], ref[l].x[0][at // PAGE, :, at % PAGE])
        if step % 5:
            cache.commit(cu, n)
            lens += q
        else:
            cache.commit(cu, n, dev(np.array([1, -1], np.int32)))
            lens += [2, 0]
        np.testing.assert_array_equal(cache.seq_len.cpu().numpy(), lens)
    used = int((cache.block_table >= 0).sum().item())
    assert used == sum(-(-int(l) // PAGE) for l in lens) and int(cache.free_count.item()) == 20 - used and int(cache.status.item()) == 0


# ---------------------------------------------------------------------------------------------------- streams, graphs, refusals
def _step(cache, cu, n, k, v, q):
    row_slot, _ = cache.reserve(cu, n)
    cache.append(k, v, row_slot)
    out = cache.attend(q, cu)
    return row_slot, out


@pytest.mark.parametrize("ctx,lens", [([3000, 40], [1, 1]), ([500, 700], [60, 130])])
def test_a_captured_step_replays(ctx, lens):
    """reserve, append and attend in one graph, replayed with new inputs and eager calls between the replays."""
    rng = np.random.default_rng(14)
    cache = make_cache(400, 2, 2, 210)
    fill(cache, rng, ctx, [0, 0], torch.bfloat16)
    cache.snapshot()
    cu, n = cu_of(lens), sum(lens)
    k, v, q = (rand_rows(rng, n, h, torch.bfloat16).cuda() for h in (2, 2, 8))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(cache, cu, n, k, v, q)
    torch.cuda.current_stream().wait_stream(side)
    cache.restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slot, out = _step(cache, cu, n, k, v, q)
    for rep in range(4):
        for t, h in ((k, 2), (v, 2), (q, 8)):
            t.copy_(rand_rows(rng, n, h, torch.bfloat16))
        cache.restore()
        graph.replay()
        torch.cuda.synchronize()
        got, got_slot, pages = out.clone(), slot.clone(), cache.k_codes.clone()
        cache.restore()
        want_slot, want = _step(cache, cu, n, k, v, q)
        assert torch.equal(got_slot, want_slot) and torch.equal(got, want) and torch.equal(pages, cache.k_codes), rep


def test_two_streams_at_once_and_the_same_bits_twice():
    rng = np.random.default_rng(15)
    work = []
    for ctx, lens in (([4000, 100, 2500], [1, 1, 1]), ([300, 900], [200, 64])):
        cache = make_cache(600, 2, 3, 300)
        fill(cache, rng, ctx, lens, torch.bfloat16)
        q = rand_rows(rng, sum(lens), 8, torch.bfloat16).cuda()
        work.append((cache, q, cu_of(lens), cache.attend(q, cu_of(lens))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    outs = [[] for _ in work]
    for _ in range(10):
        for i, (cache, q, cu, _) in enumerate(work):
            with torch.cuda.stream(streams[i]):
                outs[i].append(cache.attend(q, cu))
    torch.cuda.synchronize()
    for (_, _, _, want), got in zip(work, outs):
        assert all(torch.equal(want, g) for g in got)


def test_python_refusals():
    cache = make_cache(8, 2, 2, 4)
    cu, slot = cu_of([1, 2]), torch.zeros(3, dtype=torch.int32, device="cuda")
    ok = torch.zeros(3, 2, HD, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 4, HD, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: cache.append(ok.half(), ok.half(), slot), lambda: cache.append(ok, ok.float(), slot), lambda: cache.append(ok.cpu(), ok, slot),
                 lambda: cache.append(ok[:2], ok, slot), lambda: cache.append(ok, ok, slot.long()), lambda: cache.append(ok, ok, slot, layer=1),
                 lambda: cache.append(ok, ok, slot, layer=-1), lambda: cache.append(ok.transpose(0, 1), ok, slot),
                 lambda: cache.append(ok[:1].expand(3, 2, HD), ok, slot), lambda: cache.append(torch.cat([ok, ok], 2)[..., ::2], ok, slot),
                 lambda: cache.read(slot, torch.float16), lambda: cache.read(slot.long()), lambda: cache.read(slot[::2]),
                 lambda: cache.attend(q[:, :3], cu), lambda: cache.attend(q[0], cu), lambda: cache.attend(q.half(), cu),
                 lambda: cache.attend(q[..., :32], cu), lambda: cache.attend(q, cu.long()), lambda: cache.attend(q, cu.cpu()),
                 lambda: cache.attend(q, cu_of([1, 1, 1])), lambda: cache.attend(q, cu, out=torch.zeros_like(q.float())),
                 lambda: cache.attend(q, cu, out=torch.zeros_like(q)[:2]), lambda: cache.attend(q, cu, seq_slot=slot),
                 lambda: cache.reserve(cu, -1), lambda: cache.reserve(cu[:1], 0), lambda: cache.commit(cu, 3, accept_len=slot)):
        with pytest.raises(ValueError):
            call()
    from paper_2602_12957_amd.binding import HsdError
    with pytest.raises(HsdError):
        cache.attend(q, cu, scale=math.inf)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,lens,heads", [([40], [3], (96, 1)), ([100, 5], [2, 3], (400, 2)), ([33], [2], (1024, 1)), ([50, 20], [9, 4], (21, 3)),
                                            ([70, 3], [5, 1], (48, 24)), ([20, 90], [3, 2], (32, 16))])
def test_attend_with_many_heads(dtype, ctx, lens, heads):
    """Query heads of a kv head over several tiles, and kv heads that are no power of two or more than eight."""
    rng = np.random.default_rng(sum(ctx) + heads[0])
    maxb = max((c + n) // PAGE + 1 for c, n in zip(ctx, lens))
    cache = make_cache(len(ctx) * maxb, heads[1], len(ctx), maxb, shuffle=3)
    fill(cache, rng, ctx, lens, dtype)
    q = rand_rows(rng, sum(lens), heads[0], dtype, 0.3).cuda()
    check_attend(cache, cache.attend(q, cu_of(lens)), q, ctx, lens, dtype)


@pytest.mark.parametrize("ctx,lens,heads", [([300, 0], [500, 330], (160, 32)), ([100], [2100], (64, 64)), ([37, 500, 9], [1000, 1, 1100], (96, 32))])
def test_attend_of_blocks_that_fill_the_chip(ctx, lens, heads):
    """2048 tiles of 64 columns and more: those are taken by a wave each.  One sequence has a page without a block."""
    rng = np.random.default_rng(sum(ctx))
    maxb = max((c + n) // PAGE + 1 for c, n in zip(ctx, lens))
    cache = make_cache(len(ctx) * maxb, heads[1], len(ctx), maxb, shuffle=4)
    fill(cache, rng, ctx, lens, torch.bfloat16)
    q = rand_rows(rng, sum(lens), heads[0], torch.bfloat16, 0.3).cuda()
    rows = set(np.cumsum([0] + lens[:-1]).tolist()) | {sum(lens) - 1, lens[0] - 1, lens[0] // 2, 63, 64}
    out = cache.attend(q, cu_of(lens))
    check_attend(cache, out, q, ctx, lens, torch.bfloat16, rows=rows)
    again = cache.attend(q, cu_of(lens))
    assert torch.equal(out, again)
    cache.block_table[0, 2] = -1
    hidden = [np.arange(32, 48) if s == 0 else np.array([], int) for s in range(len(ctx))]
    # (the values are read before: a hidden block has no place to read them from)
    got = cache.attend(q, cu_of(lens))
    cache.block_table[0, 2] = 0
    check_attend(cache, got, q, ctx, lens, torch.bfloat16, rows=rows, hidden=hidden)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_and_rows_beyond_32_bits(dtype):
    """Codes of 4.5 GB each, in pages whose offsets differ by 2^32; rows of k, v, q and out that lie 2^30 elements apart."""
    rng = np.random.default_rng(12)
    ctx, lens = [70, 33], [1, 2]
    cache = make_cache(1100000, 4, 2, 8)
    far = (1 << 32) // (4 * 1024)       # blocks from one offset to the next that agrees in 32 bits
    ids = [[i, i + far] for i in (0, 1, 7, 50000)]
    ids = [b for pair in ids for b in pair] + [cache.n_blocks - 1, cache.n_blocks - 2]
    cache.free_list[-len(ids):] = dev(np.array(ids[::-1], np.int32))
    fill(cache, rng, ctx, lens, dtype)
    assert set(cache.block_table[cache.block_table >= 0].tolist()) <= set(ids) and int((cache.block_table >= 0).sum()) >= 8
    want = [sequence_values(cache, s, c + n) for s, (c, n) in enumerate(zip(ctx, lens))]
    assert all(np.abs(w).sum() > 0 for w in want)
    apart = (1 << 30) + 16
    wide = torch.empty(2 * apart + 4096, dtype=dtype, device="cuda")
    rows = rand_rows(rng, 3, 4, dtype).cuda()
    k = wide.as_strided((3, 4, HD), (apart, HD, 1))
    k.copy_(rows)
    slots, _ = cache.reserve(cu_of(lens), 3)
    cache.append(k, k, slots)           # (the rows of the block once more, with other values)
    got = cache.read(slots, torch.float32)[0]     # half a step of the largest value that the pages hold, earlier tokens included
    most = max(np.abs(w[0]).max() for w in want + [rows.float().cpu().numpy()[None]])
    assert (got - rows.float()).abs().max() <= 2.0 ** -4 * most
    q = rand_rows(rng, 3, 16, dtype, 0.3).cuda()
    wide_q = wide.as_strided((3, 16, HD), (apart, HD, 1))
    wide_q.copy_(q)
    out = torch.empty_like(wide).as_strided((3, 16, HD), (apart, HD, 1))
    cache.attend(wide_q, cu_of(lens), out=out)
    check_attend(cache, out.contiguous(), q, ctx, lens, dtype)
