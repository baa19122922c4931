"""Scores of given tokens against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, tokens, n_top):
    """x: fp64 [rows, vocab] -> logprob, entropy, ids, logprobs (the definition, row by row)"""
    lp, ent = np.empty(len(x)), np.empty(len(x))
    ids, tl = np.full((len(x), n_top), -1, np.int32), np.full((len(x), n_top), -np.inf)
    for r, row in enumerate(x):
        t = int(tokens[r])
        inside = 0 <= t < len(row)
        order = np.argsort(np.where(np.isnan(row), np.inf, -row), kind="stable")
        order = order[(row[order] > -np.inf)][:n_top]
        ids[r, :len(order)] = order
        if np.isnan(row).any() or (row == np.inf).any():
            lp[r], ent[r], tl[r, :len(order)] = (np.nan if inside else -np.inf), np.nan, np.nan
            continue
        m = row.max()
        if m == -np.inf:
            lp[r], ent[r] = -np.inf, 0.0
            continue
        z = np.exp(row - m).sum()
        logp = row - m - np.log(z)
        p = np.exp(logp)
        lp[r] = logp[t] if inside else -np.inf
        ent[r] = -(p[p > 0] * logp[p > 0]).sum()
        tl[r, :len(order)] = logp[order]
    return lp, ent, ids, tl


def check(logits, tokens, n_top, got=None):
    from paper_2602_12957_amd.scoring import token_logprobs
    got = token_logprobs(logits, tokens, n_top) if got is None else got
    x = logits.double().cpu().numpy()
    lp, ent, ids, tl = reference(x, tokens.cpu().numpy(), n_top)
    np.testing.assert_array_equal(got.top_ids.cpu().numpy(), ids)
    # Roundings (2^-24 each, relative).  Z: an exponential (its argument to half a step of |x - m| <= 104, where it is not 0:
    # 104 roundings; 4 of its own) and the sums (1024 in a row within a thread, 32 of joining and rescaling); its logarithm then moves by as
    # much, absolutely, and by 2 roundings of itself; x - m and the difference by one of their magnitudes each.  Entropy: ln Z and
    # W / Z, whose terms add what |x - m| <= 104 weighs: the same relative error of W's magnitude sum.
    u = 2.0 ** -24
    dz = (104 + 4 + 1024 + 32) * u
    with np.errstate(invalid="ignore", over="ignore"):
        for g, want in ((got.logprob, lp), (got.top_logprobs, tl)):
            want = want.astype(np.float32).astype(np.float64)      # a difference may be beyond the type
            g = g.double().cpu().numpy()
            fin = np.isfinite(want)
            np.testing.assert_array_equal(g[~fin], want[~fin])
            assert (np.abs(g - want)[fin] <= dz + 4 * u * np.abs(want[fin]) + 4 * u * 12).all(), np.abs(g - want)[fin].max()
        g = got.entropy.double().cpu().numpy()
        fin = np.isfinite(ent)
        np.testing.assert_array_equal(np.isnan(g), ~fin)
        assert (np.abs(g - ent)[fin] <= 2 * dz * (1 + ent[fin]) + 8 * u * 12).all(), np.abs(g - ent)[fin].max()


def make(rng, rows, vocab, dtype, spread=2.0):
    x = spread * rng.standard_normal((rows, vocab))
    x[np.arange(rows), rng.integers(0, vocab, rows)] += rng.uniform(0, 12, rows)
    return torch.from_numpy(x).to(dtype).cuda(), torch.from_numpy(rng.integers(0, vocab, rows).astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 32768, 5), (3, 5, 8), (16, 32749, 20), (2, 151936, 32), (7, 1000, 0), (33, 4096, 1), (5, 63, 32), (1, 8193, 32),
                                            (300, 2049, 8), (130, 32768, 3), (2, 262145, 1), (600, 12345, 32)])
def test_token_logprobs_against_the_definition(dtype, rows, vocab, top):
    rng = np.random.default_rng(rows + vocab)
    logits, tokens = make(rng, rows, vocab, dtype)
    check(logits, tokens, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [40, 5000, 70001])
def test_masks_ties_and_values_that_are_not_finite(dtype, vocab):
    rng = np.random.default_rng(vocab)
    low = torch.finfo(dtype).min
    x = 2.0 * rng.standard_normal((16, vocab))
    x[0] = -np.inf                                   # nothing is left
    x[1] = -np.inf; x[1, vocab - 3] = 4.0            # one token
    x[2] = 1.25                                      # all alike: the lowest ids
    x[3] = low                                       # a mask of the type's lowest value, everywhere
    x[4] = low; x[4, [7, 11]] = [0.5, 0.5]           # .. and two tokens
    x[5, ::2] = -np.inf
    x[6] = np.round(x[6])                            # many ties
    x[7, vocab // 2] = np.nan
    x[8, 3] = np.inf
    x[9, vocab - 1] = -torch.finfo(dtype).min        # the largest number; below it the lowest
    x[9, :5] = low
    x[10] = np.linspace(-50, 50, vocab)              # rising: every tile moves the maximum
    x[11] = np.linspace(50, -50, vocab)
    x[12, :] = -np.inf; x[12, 5] = np.nan
    x[13] = 88.0 * np.sign(x[13])
    x[14] = 0.0; x[14, vocab // 3] = 200.0           # certain
    x[15] = -np.inf; x[15, [1, vocab - 1]] = [np.inf, 2.0]
    logits = torch.from_numpy(x).to(dtype).cuda()
    tokens = torch.from_numpy(rng.integers(0, vocab, 16).astype(np.int32)).cuda()
    tokens[1], tokens[4], tokens[5], tokens[14] = vocab - 3, 7, 2, vocab // 3
    for top in (0, 1, 6, 32):
        check(logits, tokens, top)
    tokens[:] = torch.tensor([-1, vocab, 1 << 30, -(1 << 31)] * 4, dtype=torch.int32)
    check(logits, tokens, 2)


def test_rows_of_a_wider_tensor_at_odd_elements():
    rng = np.random.default_rng(3)
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.from_numpy(rng.standard_normal((9, 5003))).to(dtype).cuda()
        wide[:, 0], wide[:, 4000:] = math.nan, math.inf          # outside
        check(wide[:, 1:3998], torch.arange(9, dtype=torch.int32, device="cuda"), 7)
        check(wide[4:5, 3:3998], torch.zeros(1, dtype=torch.int32, device="cuda"), 7)


def test_no_rows_and_refusals():
    from paper_2602_12957_amd.scoring import token_logprobs
    x, t = torch.zeros((3, 50), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    r = token_logprobs(x[:0], t[:0], 4)
    assert r.logprob.shape == (0,) and r.top_ids.shape == (0, 4)
    for call in (lambda: token_logprobs(x.half(), t), lambda: token_logprobs(x.cpu(), t.cpu()), lambda: token_logprobs(x, t.long()),
                 lambda: token_logprobs(x, t[:2]), lambda: token_logprobs(x, t, -1), lambda: token_logprobs(x, t, 33), lambda: token_logprobs(x.t(), t),
                 lambda: token_logprobs(x[0], t), lambda: token_logprobs(x[:, :0], t), lambda: token_logprobs(x[:1].expand(3, 50), t),
                 lambda: token_logprobs(x, t.cpu())):
        with pytest.raises(ValueError):
            call()


def test_a_captured_call_replays_and_two_streams_agree():
    from paper_2602_12957_amd.scoring import token_logprobs
    rng = np.random.default_rng(4)
    logits, tokens = make(rng, 20, 32768, torch.float32)
    token_logprobs(logits, tokens, 9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = token_logprobs(logits, tokens, 9)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(4):
        logits.copy_(make(rng, 20, 32768, torch.float32)[0])
        graph.replay()
        torch.cuda.synchronize()
        have = [g.clone() for g in got]
        check(logits, tokens, 9, got)
        outs = []
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(token_logprobs(logits, tokens, 9))
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o, have)), rep


@pytest.mark.parametrize("dtype,step", [(torch.bfloat16, 512), (torch.float32, 256)])
@pytest.mark.parametrize("rows", [2, 700])
def test_large_logits_64_pieces_apart(dtype, step, rows):
    """The largest logits at one lane's places: more of them reach the bound than the list holds."""
    rng = np.random.default_rng(6)
    vocab = 40 * step + 3
    x = rng.standard_normal((rows, vocab))
    for e in range(step // 64):
        for lane in range(32):
            x[:, lane * (step // 64) + e::step] += 30.0 + 0.001 * lane
    logits = torch.from_numpy(x).to(dtype).cuda()
    check(logits, torch.zeros(rows, dtype=torch.int32, device="cuda"), 32)
    check(logits, torch.zeros(rows, dtype=torch.int32, device="cuda"), 5)


@pytest.mark.parametrize("dtype,line", [(torch.bfloat16, 64), (torch.float32, 32)])
@pytest.mark.parametrize("rows,turns", [(3, 12), (600, 5), (1100, 5)])
def test_large_logits_64_lines_apart(dtype, line, rows, turns):
    """The largest logits in the lines of half of the groups: more of them reach the bound than the list holds."""
    rng = np.random.default_rng(8)
    vocab = turns * 64 * line + 5
    x = rng.standard_normal((rows, vocab))
    where = (np.arange(vocab) // line) % 2 == 0
    x[:, where] += 40.0
    logits = torch.from_numpy(x).to(dtype).cuda()
    tokens = torch.from_numpy(rng.integers(0, vocab, rows).astype(np.int32)).cuda()
    check(logits, tokens, 32)
    check(logits, tokens, 5)


def test_many_rows():
    """More rows than a grid's second dimension takes."""
    rng = np.random.default_rng(7)
    logits, tokens = make(rng, 70000, 40, torch.float32)
    check(logits, tokens, 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_beyond_32_bits(dtype):
    """Rows that lie 2^30 elements apart."""
    rng = np.random.default_rng(13)
    logits, tokens = make(rng, 3, 1000, dtype)
    apart = (1 << 30) + 3
    wide = torch.empty(2 * apart + 1000, dtype=dtype, device="cuda").as_strided((3, 1000), (apart, 1))
    wide.copy_(logits)
    check(wide, tokens, 4)
