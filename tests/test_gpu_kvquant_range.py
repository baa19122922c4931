"""Attention over the 8-bit cache where its running reference moves: scores that rise by tens to hundreds of binary orders after a
wave's first step, in every form of the kernel, against the definition in 64 bits.

A wave walks every W-th pair of pages of its run.  FORMS are sized so that the keys in question lie in its second step or later: 64
columns are one wave's, the others have 16 (bf16) or 8 (fp32) at most."""
import math

import numpy as np
import pytest
import torch

from test_gpu_kvquant import EPS, HD, PAGE, check_attend, cu_of, make_cache

pytestmark = pytest.mark.gpu

# type, cached tokens, rows, (query heads, kv heads), entries of the block table (None: as many as are needed; above 256 the keys are
# split over workgroups)
FORMS = {"64 columns, a row a half": (torch.bfloat16, 700, 2100, (64, 2), None),
         "64 columns, eight rows a half": (torch.bfloat16, 700, 2100, (64, 16), None),
         "32 columns, one row": (torch.bfloat16, 3000, 1, (16, 4), None),
         "32 columns, a block": (torch.bfloat16, 1500, 70, (16, 4), None),
         "32 columns, split keys": (torch.bfloat16, 9000, 20, (16, 4), 600),
         "two parts, split keys": (torch.bfloat16, 9000, 1, (16, 4), 600),
         "fp32, one row": (torch.float32, 3000, 1, (16, 4), None),
         "fp32, a block": (torch.float32, 1500, 70, (16, 4), None),
         "fp32, split keys": (torch.float32, 9000, 1, (16, 4), 600)}


def place(cache, k, v, ctx, n):
    """One sequence: ctx cached tokens and n rows behind them, whose blocks are taken and which are not committed."""
    for a, b in ((0, ctx), (ctx, ctx + n)):
        cu = cu_of([b - a])
        slots, _ = cache.reserve(cu, b - a)
        cache.append(k[a:b].cuda(), v[a:b].cuda(), slots)
        if b == ctx:
            cache.commit(cu, ctx)
    assert int(cache.status.item()) == 0


def setup(form, seed):
    dtype, ctx, n, heads, maxb = FORMS[form]
    rng = np.random.default_rng(seed)
    cache = make_cache((ctx + n) // PAGE + 2, heads[1], 1, maxb or (ctx + n) // PAGE + 1, shuffle=seed)
    k, v = (rng.standard_normal((ctx + n, heads[1], HD)) for _ in range(2))
    q = 0.3 * rng.standard_normal((n, heads[0], HD))
    k[:, :, 0] = q[:, :, 0] = 0.0
    return dtype, ctx, n, heads, cache, rng, k, v, q


def looked_at(rng, n):
    """Rows to compare: the first ones, both sides of the middle, the last ones, and some."""
    return set(range(n)) if n <= 2 else {0, 1, 4, n // 2, n - 1} | set(rng.integers(0, n, 3).tolist())


# which columns (row * heads of the group + head) meet the keys that stand out
COLUMNS = {"all": lambda f: f >= 0, "first half": lambda f: f // 32 % 2 == 0, "second half": lambda f: f // 32 % 2 == 1,
           "two sixteen apart": lambda f: np.isin(f % 32, (5, 21)), "one": lambda f: f % 64 == 37}


@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("orders", [30, 60, 100, 200])
@pytest.mark.parametrize("form", FORMS)
def test_scores_that_jump_within_the_walk(form, orders, order):
    """Keys in the middle, at the end and among the block's own exceed all others by `orders` binary orders and more."""
    dtype, ctx, n, heads, cache, rng, k, v, q = setup(form, orders)
    group = heads[0] // heads[1]
    late, own = (20.0, 26.0) if order == "rising" else (10.0, 8.0)
    for at, height in ((ctx // 2, 16.0), (ctx // 2 + 3, 16.0), (ctx - 5, late), (ctx - 45, late), (ctx + n // 2 if n > 1 else ctx - 70, own)):
        k[at, :, 0] = height
    k, v = (torch.from_numpy(x).to(dtype) for x in (k, v))
    place(cache, k, v, ctx, n)
    f = np.arange(n)[:, None] * group + np.arange(heads[0])[None] % group
    for name in COLUMNS if group * n > 4 else ["all"]:
        x = q.copy()
        x[:, :, 0] = np.where(COLUMNS[name](f), orders / (0.125 * 16.0 * math.log2(math.e)), 0.0)
        x = torch.from_numpy(x).to(dtype).cuda()
        out = cache.attend(x, cu_of([n]))
        assert bool(torch.isfinite(out).all()), name
        check_attend(cache, out, x, [ctx], [n], dtype, rows=looked_at(rng, n))


@pytest.mark.parametrize("length", [20 * PAGE, 20 * PAGE + 5, (1 << 31) - 1, (1 << 31) - 40])
def test_a_length_that_no_table_holds(length):
    """Such a sequence has no place for rows, which is reported, and sees the whole table; the one beside it stays as it is."""
    rng = np.random.default_rng(3)
    cache = make_cache(41, 2, 2, 20)
    x = torch.from_numpy(rng.standard_normal((2 * 20 * PAGE, 2, HD))).to(torch.bfloat16).cuda()
    full = cu_of([20 * PAGE] * 2)
    slots, _ = cache.reserve(full, 2 * 20 * PAGE)
    cache.append(x, x.flip(0), slots)
    q, cu = torch.from_numpy(0.3 * rng.standard_normal((53, 8, HD))).to(torch.bfloat16).cuda(), cu_of([50, 3])
    cache.seq_len[0], cache.seq_len[1] = 20 * PAGE, 200
    want = cache.attend(q, cu)
    cache.seq_len[0] = length
    table = cache.block_table.clone()
    assert torch.equal(cache.attend(q, cu), want)
    slots, pos = cache.reserve(cu, 53)
    assert int(cache.status.item()) == 2 and int(cache.free_count.item()) == 1 and torch.equal(cache.block_table, table)
    assert bool((slots[:50] == -1).all()) and bool((slots[50:] >= 0).all()) and pos[50:].tolist() == [200, 201, 202]
    cache.commit(cu, 53, torch.tensor([45, 1], dtype=torch.int32, device="cuda"))
    assert int(cache.seq_len[1].item()) == 202 and int(cache.free_count.item()) == 1 and torch.equal(cache.block_table, table)


@pytest.mark.parametrize("orders", [0, 100])
@pytest.mark.parametrize("where", ["everywhere", "late page", "one key"])
@pytest.mark.parametrize("form", FORMS)
def test_values_up_to_the_largest_that_a_page_holds(form, where, orders):
    """Averages are finite where sums over the keys are not; keys that stand out by 100 orders let those of 2^127 in at 2^-100."""
    dtype, ctx, n, heads, cache, rng, k, v, q = setup(form, orders + 1)
    k[[ctx // 2, ctx // 2 + 40], :, 0] = 16.0
    q[:, :, 0] = orders / (0.125 * 16.0 * math.log2(math.e))
    most = math.ldexp(448.0, 119)
    at = {"everywhere": slice(None), "late page": slice((ctx - 20) // PAGE * PAGE, (ctx - 20) // PAGE * PAGE + PAGE), "one key": slice(ctx // 2 + 40, ctx // 2 + 41)}[where]
    v[at] = np.sign(v[at]) * np.ldexp(1.0, rng.integers(90, 128, v[at].shape))
    v[at, :, 5], v[at, :, 6] = most, -most
    k, v = (torch.from_numpy(x).to(dtype) for x in (k, v))
    place(cache, k, v, ctx, n)
    x = torch.from_numpy(q).to(dtype).cuda()
    out = cache.attend(x, cu_of([n]))
    assert bool(torch.isfinite(out).all())
    check_attend(cache, out, x, [ctx], [n], dtype, rows=looked_at(rng, n))


def two_key_case(seed):
    """One row of 16 heads over 5000 keys of which two count, by nearly equal probabilities, with values that nearly cancel."""
    rng = np.random.default_rng(seed)
    cache = make_cache(320, 4, 1, 320)
    k, v = np.zeros((5000, 4, HD)), rng.standard_normal((5000, 4, HD))
    q = np.zeros((1, 16, HD))
    k[:, :, 0], q[:, :, 0] = -16.0, 16.0      # 64 natural units below the two
    k[[2000, 2010], :, 0] = 16.0
    k[2010, :, 1], q[0, :, 1] = 1.0, -np.linspace(0.01, 0.9, 16)
    v[2000], v[2010] = 1.0, -1.0
    k, v, q = (torch.from_numpy(x).to(torch.bfloat16) for x in (k, v, q))
    place(cache, k, v, 4999, 1)
    return cache, q


def test_probabilities_of_single_tokens_on_split_keys_carry_16_bits():
    """o = (1 - p) / (1 + p): with p in one bf16 part it would be off by up to 2^-9 of the spread, which is 1; with two by 2^-17 at
    most.  That the case tells the two apart is worked out from the rounding of p alone."""
    cache, q = two_key_case(21)
    out = cache.attend(q.cuda(), cu_of([1])).double().cpu().numpy()[0]
    x = q.double().numpy()[0, :, 1] * 0.125
    p = np.exp(x)
    want = (1.0 - p) / (1.0 + p)
    # two parts: 2^-16 of p; fp32: the score's two products and their sum (4 roundings of 256, times 0.125), exponent, exponential and
    # sums (8 each), for both keys; the output's own half step
    tol = 2.0 ** -16 + 2.0 ** -24 * 2 * (4 * 32 + 24) + EPS[torch.bfloat16] * np.abs(want)
    one = torch.from_numpy(p).to(torch.bfloat16).double().numpy()
    assert (np.abs((1.0 - one) / (1.0 + one) - want) > tol).sum() >= 8
    assert (np.abs(out - want[:, None]) <= tol[:, None]).all(), float((np.abs(out - want[:, None]) / tol[:, None]).max())
