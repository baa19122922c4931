"""The operators around a cache that is held in 8 bits, as calls that can be timed and compared.

A serving step on such a cache places the new rows of every sequence in pages (`QuantKV.reserve`), quantises their keys and
values into them (`append`), lets their queries attend to the pages (`attend`) and, behind the LM head, scores tokens
(`token_logprobs`).  A page holds 16 tokens of one kv head as e4m3 codes with one power-of-two scale for its keys and one for
its values: the smallest 2^e with 448 * 2^e >= the largest magnitude of the page.

With `own` false the operators run in plain torch, 32 bits, rounded once at the end.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False
DEV = "cuda:0"
PAGE, HD = 16, 64
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # rows of 16 regions that decode side by side: the smallest placing
        dict(name="place_step_16", op="place", n_seq=16, ctx=1055, q=1, q_hi=1, shape=3),
        # the first round of 64 ragged regions
        dict(name="place_ragged_64", op="place", n_seq=64, ctx=512, ctx_hi=2048, q=8, q_hi=256, shape=5),
        # one new token of 64 sequences
        dict(name="append_step_64", op="append", n_seq=64, ctx=512, ctx_hi=2048, q=1, q_hi=1, n_kv=4, dtype="bf16", shape=7),
        # four pages of 8193 rows behind prefixes that end inside a page
        dict(name="append_page_4", op="append", n_seq=4, ctx=8188, ctx_hi=8197, q=8193, q_hi=8193, n_kv=4, dtype="bf16", shape=9),
        # one user, one token: the latency of the smallest attention
        dict(name="attend_step_1", op="attend", n_seq=1, ctx=1055, q=1, q_hi=1, n_q=16, n_kv=4, dtype="bf16", shape=11),
        # one token of 64 sequences whose prefixes differ in length
        dict(name="attend_step_64", op="attend", n_seq=64, ctx=512, ctx_hi=2048, q=1, q_hi=1, n_q=16, n_kv=4, dtype="bf16", shape=13),
        # one token of eight sequences over very long caches
        dict(name="attend_long_8", op="attend", n_seq=8, ctx=131072, ctx_hi=131071 + 37, q=1, q_hi=1, n_q=16, n_kv=4, dtype="bf16", shape=15),
        # the drafts of a page's 16 regions
        dict(name="attend_region_16", op="attend", n_seq=16, ctx=1055, q=17, q_hi=257, n_q=16, n_kv=4, dtype="bf16", shape=17),
        # one long draft of four pages each over a prefix of the same length: the largest call
        dict(name="attend_page_4", op="attend", n_seq=4, ctx=8192, q=8193, q_hi=8193, n_q=16, n_kv=4, dtype="bf16", shape=19),
        # the small fp32 model, every head with keys of its own
        dict(name="attend_fp32_4", op="attend", n_seq=4, ctx=271, q=33, q_hi=33, n_q=4, n_kv=4, dtype="fp32", shape=21),
        # scores of the tokens that 16 sequences decoded, five alternatives each
        dict(name="score_step_16", op="score", rows=16, vocab=32768, pad=0, top=5, masked=0.0, dtype="fp32"),
        # scores of a whole round of drafts, logits of a padded head
        dict(name="score_draft_1856", op="score", rows=1856, vocab=32749, pad=19, top=8, masked=0.02, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["place", "append", "append", "attend", "attend", "attend", "block", "block", "score", "score"])
    shape = rng.randrange(1 << 20)
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "place":
        n = _log(rng, 1, 2048)
        lo, q = _log(rng, 1, 8192), _log(rng, 1, max(2, 16384 // n)) - 1
        return dict(op="place", n_seq=n, ctx=lo, ctx_hi=2 * lo, q=q, q_hi=2 * q + 1, shape=shape)
    if op == "append":
        n, n_kv = _log(rng, 1, 64), rng.choice([1, 2, 3, 4, 8])
        q = _log(rng, 1, max(2, 32768 // n // n_kv))
        lo = _log(rng, 1, 4096)
        return dict(op="append", n_seq=n, ctx=lo, ctx_hi=2 * lo, q=q, q_hi=q if q < 4 else q + q // 4, n_kv=n_kv, dtype=dtype, shape=shape)
    if op == "attend":
        n = _log(rng, 1, 64)
        n_q, n_kv = rng.choice([(16, 4), (4, 4), (8, 2), (32, 8), (12, 4), (16, 2), (6, 2), (5, 1)])
        lo = _log(rng, 1, min(98304, (1 << 21) // n // n_kv))
        return dict(op="attend", n_seq=n, ctx=lo, ctx_hi=lo + lo // 2, q=1, q_hi=rng.choice([1, 1, 4, 8]), n_q=n_q, n_kv=n_kv, dtype=dtype, shape=shape)
    if op == "block":
        n = _log(rng, 1, 16)
        n_q, n_kv = rng.choice([(16, 4), (4, 4), (8, 2), (12, 4), (16, 2), (6, 2)])
        q, lo = _log(rng, 2, 8192 // n if dtype == "bf16" else 2048 // n), _log(rng, 1, 4096)
        return dict(op="attend", n_seq=n, ctx=lo, ctx_hi=2 * lo, q=q, q_hi=q + q // 2, n_q=n_q, n_kv=n_kv, dtype=dtype, shape=shape)
    vocab = _log(rng, 500, 200000)
    return dict(op="score", rows=_log(rng, 1, max(2, min(4096, 48000000 // vocab))), vocab=vocab, pad=rng.choice([0, 0, 1, 64]),
                top=rng.choice([0, 1, 5, 8, 20, 32]), masked=rng.choice([0.0, 0.0, 0.5, 0.999]), dtype=rng.choice(["bf16", "fp32"]), shape=shape)


def _lens(case):
    """(cached tokens, new rows) of every sequence; they follow from the case alone."""
    rng = random.Random(case["shape"])
    ctx = [rng.randint(case["ctx"], case.get("ctx_hi", case["ctx"])) for _ in range(case["n_seq"])]
    q = [rng.randint(case["q"], case["q_hi"]) for _ in ctx]
    if sum(q) == 0:
        q[0] = 1
    return ctx, q


def work(case):
    if case["op"] == "score":
        es = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["vocab"]
        return {"bytes": n * es + case["rows"] * (12 + 8 * case["top"]), "flops": 6 * n}
    ctx, q = _lens(case)
    rows, pages = sum(q), sum((c + k + PAGE - 1) // PAGE - c // PAGE for c, k in zip(ctx, q))
    if case["op"] == "place":
        return {"bytes": 12 * case["n_seq"] + 8 * rows + 8 * pages, "flops": 2 * rows}
    es, n_kv = 2 if case["dtype"] == "bf16" else 4, case["n_kv"]
    if case["op"] == "append":   # rows in, codes and scales out, and the values read back
        kept = sum(c % PAGE for c, k in zip(ctx, q) if k)
        return {"bytes": 2 * n_kv * ((rows + kept) * HD * (es + 2) + rows * HD * es + 8 * pages), "flops": 6 * rows * n_kv * HD}
    n_q = case["n_q"]
    seen = sum(k * c + k * (k + 1) // 2 for c, k in zip(ctx, q))
    keys = sum(c + k for c, k in zip(ctx, q) if k)
    return {"bytes": 2 * rows * n_q * HD * es + keys * n_kv * 2 * HD + keys * n_kv // 2, "flops": 4 * HD * n_q * seen}


# ---------------------------------------------------------------------------------------------------- plain cache
def _exponent(amax):
    """Smallest e in [-100, 119] with 448 * 2^e >= amax, as an integer tensor; 0 where amax is 0."""
    m, x = torch.frexp(amax.float())          # amax = m * 2^x, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e.clamp(-100, 119), torch.zeros_like(e))


class PlainKV:
    """Pages as [block, kv head, token, dim] e4m3 values and one scale a page."""

    def __init__(self, n_blocks, n_kv):
        self.codes = [torch.zeros((n_blocks, n_kv, PAGE, HD), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
        self.scale = [torch.ones((n_blocks, n_kv), dtype=torch.float32, device=DEV) for _ in range(2)]

    def append(self, k, v, slots):
        slots = slots.long()
        blk, off = slots // PAGE, slots % PAGE
        pages, at = torch.unique(blk, return_inverse=True)
        first = torch.full((len(pages),), PAGE, dtype=torch.long, device=DEV).scatter_reduce(0, at, off, "amin")
        kept = (torch.arange(PAGE, device=DEV)[None] < first[:, None])[:, None, :, None]
        for i, x in enumerate((k, v)):
            page = self.codes[i][pages].float() * self.scale[i][pages][:, :, None, None]
            page = torch.where(kept, page, torch.zeros_like(page))
            page[at, :, off] = x.float()
            e = _exponent(page.abs().amax((2, 3)))
            s = ((e.int() + 127) << 23).view(torch.float32)   # 2^e, by its bits: pow rounds
            self.codes[i].view(torch.uint8)[pages] = (page / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            self.scale[i][pages] = s

    def rows(self, i, slots):
        slots = slots.long()
        return self.codes[i].view(torch.uint8)[slots // PAGE, :, slots % PAGE].view(torch.float8_e4m3fn).float() * self.scale[i][slots // PAGE][..., None]

    def sequence(self, i, pages, n):
        x = self.codes[i].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() * self.scale[i][pages][:, :, None, None]
        return x.transpose(0, 1).reshape(x.shape[1], -1, HD)[:, :n]


def _plain_place(s):
    """Tables, free ids and slots in elementary steps: count what each sequence lacks, give out ids in order, look rows up."""
    table, cu, ctx = s.table.clone(), s.cu.long(), s.ctx.long()
    lens = cu[1:] - cu[:-1]
    idx = torch.arange(table.shape[1], device=DEV)[None]
    need = (idx >= (ctx // PAGE)[:, None]) & (idx < ((ctx + lens + PAGE - 1) // PAGE)[:, None]) & (table < 0)
    rank = torch.cumsum(need.reshape(-1).int(), 0).reshape(need.shape) - 1
    n_free = s.free_count.long()
    ids = s.free_list[(n_free - 1 - rank).clamp(min=0).long()]
    table = torch.where(need, ids, table)
    seq = torch.repeat_interleave(torch.arange(len(ctx), device=DEV), lens, output_size=s.total)
    pos = ctx[seq] + torch.arange(s.total, device=DEV) - cu[seq]
    slot = table[seq, pos // PAGE].long() * PAGE + pos % PAGE
    return {"row_slot": slot.int(), "row_pos": pos.int(), "table": table, "free_count": (n_free - need.sum()).int()}


def _plain_attend(s):
    group = s.n_q // s.n_kv
    out = torch.empty((s.total, s.n_q, HD), dtype=s.dtype, device=DEV)
    r0 = 0
    for i, (c, n) in enumerate(zip(s.ctx_host, s.q_host)):
        if n == 0:
            continue
        keys = c + n
        pages = s.table[i, :(keys + PAGE - 1) // PAGE].long()
        k, v = (s.plain.sequence(j, pages, keys) for j in range(2))
        q = s.q[r0:r0 + n].float().reshape(n, s.n_kv, group, HD).transpose(0, 1)
        step = max(1, (1 << 27) // (keys * s.n_q))
        for a in range(0, n, step):
            b = min(n, a + step)
            qq = q[:, a:b].reshape(s.n_kv, (b - a) * group, HD)
            sc = torch.matmul(qq, k.transpose(1, 2)) * (1.0 / math.sqrt(HD))
            row = torch.arange(a, b, device=DEV).repeat_interleave(group)
            sc = sc.masked_fill(torch.arange(keys, device=DEV)[None] > c + row[:, None], -math.inf)
            p = torch.exp(sc - sc.amax(-1, keepdim=True))
            o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
            out[r0 + a:r0 + b] = o.reshape(s.n_kv, b - a, group, HD).transpose(0, 1).reshape(b - a, s.n_q, HD).to(s.dtype)
        r0 += n
    return out


def _plain_score(s):
    x = s.logits.float()
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(-1)
    lz = torch.log(z)
    logprob = d.gather(1, s.tokens.long()[:, None])[:, 0] - lz
    entropy = lz - torch.where(e > 0, d * e, torch.zeros_like(e)).sum(-1) / z
    out = {"logprob": logprob, "entropy": entropy}
    if s.top:
        val, idx = torch.sort(d, dim=-1, descending=True, stable=True)
        val, idx = val[:, :s.top], idx[:, :s.top]
        if val.shape[1] < s.top:
            val = torch.nn.functional.pad(val, (0, s.top - val.shape[1]), value=-math.inf)
            idx = torch.nn.functional.pad(idx, (0, s.top - idx.shape[1]), value=-1)
        gone = val == -math.inf
        out["top_ids"] = torch.where(gone, torch.full_like(idx, -1), idx).int()
        out["top_logprobs"] = val - lz[:, None]
    return out


# ---------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _kv_rows(g, n, n_kv, dtype, gain):
    """Rows whose channels differ in size, as those of trained decoders do."""
    return (torch.randn((n, n_kv, HD), generator=g, device=DEV) * gain).to(dtype)


def _kv_inputs(case, seed):
    """Keys and values of the cached tokens and of the new rows, sequence after sequence."""
    ctx, q = _lens(case)
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    gains = [torch.exp(0.7 * torch.randn((case["n_kv"], HD), generator=g, device=DEV)) for _ in range(2)]
    old = [_kv_rows(g, sum(ctx), case["n_kv"], dt, x) for x in gains]
    new = [_kv_rows(g, sum(q), case["n_kv"], dt, x) for x in gains]
    return g, ctx, q, old, new


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=DEV)


def _score_inputs(case, seed):
    g = _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    x = 2.0 * torch.randn((rows, vocab + case["pad"]), generator=g, device=DEV)
    best = torch.randint(vocab, (rows,), generator=g, device=DEV)
    x[torch.arange(rows, device=DEV), best] += 12.0 * torch.rand((rows,), generator=g, device=DEV)   # from sure to open
    logits = x.to(DTYPES[case["dtype"]])[:, :vocab]
    if case["masked"]:   # ids that a grammar or a padded vocabulary rules out
        gone = torch.rand((rows, vocab), generator=g, device=DEV) < case["masked"]
        gone[torch.arange(rows, device=DEV), best] = False
        logits.masked_fill_(gone, -math.inf)
    other = torch.randint(vocab, (rows,), generator=g, device=DEV)
    return logits, torch.where(torch.rand((rows,), generator=g, device=DEV) < 0.7, best, other).int()


def prepare(case, seed):
    s = SimpleNamespace(op=case["op"])
    if s.op == "score":
        s.logits, s.tokens = _score_inputs(case, seed)
        s.top = case["top"]
        if own:
            from paper_2602_12957_amd.scoring import token_logprobs
            s.call = token_logprobs
        return s

    if s.op == "place":
        ctx, q = _lens(case)
        g, n_kv = _gen(seed), 1
    else:
        g, ctx, q, old, new = _kv_inputs(case, seed)
        n_kv, s.dtype = case["n_kv"], DTYPES[case["dtype"]]
    s.ctx_host, s.q_host, s.total = ctx, q, sum(q)
    s.cu = _cu(q)
    n, width = case["n_seq"], max((c + k + PAGE - 1) // PAGE for c, k in zip(ctx, q)) + 1
    have = [(c + PAGE - 1) // PAGE for c in ctx]
    n_blocks = sum(have) + sum(q) // PAGE + 2 * n
    ids = torch.randperm(n_blocks, generator=g, device=DEV).int()   # a pool that has been in use for a while
    table = torch.full((n, width), -1, dtype=torch.int32)
    at, ids_host = 0, ids.cpu()
    for i, b in enumerate(have):
        table[i, :b] = ids_host[at:at + b]
        at += b
    s.table, s.ctx = table.to(DEV), torch.tensor(ctx, dtype=torch.int32, device=DEV)
    s.free_count = torch.tensor(n_blocks - at, dtype=torch.int32, device=DEV)
    s.free_list = torch.cat([ids[at:], torch.full((at,), -1, dtype=torch.int32, device=DEV)])
    if own:
        from paper_2602_12957_amd.kvquant import QuantKV
        s.kv = QuantKV(n_blocks, n_kv, n, width, device=DEV)
        s.kv.block_table.copy_(s.table)
        s.kv.seq_len.copy_(s.ctx)
        s.kv.free_list.copy_(s.free_list)
        s.kv.free_count.copy_(s.free_count.reshape(1))
    if s.op == "place":
        if own:
            s.kv.snapshot()
        return s

    # cached tokens, then the places of the new rows
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(ctx, device=DEV), output_size=sum(ctx))
    pos = torch.arange(sum(ctx), device=DEV) - _cu(ctx).long()[seq]
    old_slots = (s.table[seq, pos // PAGE] * PAGE + pos % PAGE).int()
    placed = _plain_place(s)
    s.slots, s.table = placed["row_slot"], placed["table"]
    cache = PlainKV(n_blocks, n_kv) if not own else s.kv
    cache.append(old[0], old[1], old_slots)
    s.k, s.v = new
    if own:
        s.kv.block_table.copy_(s.table)
    else:
        s.plain = cache
    if s.op == "append":
        # what the call can change: the new rows and the tokens that share a page with them
        shared = [torch.arange(c - c % PAGE, c, device=DEV) for c in ctx]
        rows = [(s.table[i, p // PAGE] * PAGE + p % PAGE).int() for i, (p, k) in enumerate(zip(shared, q)) if k]
        s.look = torch.cat(rows + [s.slots])
        return s
    s.n_q, s.n_kv = case["n_q"], n_kv
    cache.append(s.k, s.v, s.slots)
    s.q = torch.randn((s.total, s.n_q, HD), generator=g, device=DEV).to(s.dtype)
    return s


def run(s):
    if s.op == "place":
        if not own:
            return _plain_place(s)
        s.kv.restore()
        row_slot, row_pos = s.kv.reserve(s.cu, s.total)
        return {"row_slot": row_slot, "row_pos": row_pos, "table": s.kv.block_table, "free_count": s.kv.free_count[0]}
    if s.op == "append":
        if not own:
            s.plain.append(s.k, s.v, s.slots)
            return [s.plain.rows(i, s.look).to(s.dtype) for i in range(2)]
        s.kv.append(s.k, s.v, s.slots)
        return list(s.kv.read(s.look, s.dtype))
    if s.op == "attend":
        return s.kv.attend(s.q, s.cu) if own else _plain_attend(s)
    if not own:
        return _plain_score(s)
    r = s.call(s.logits, s.tokens, s.top)
    out = {"logprob": r.logprob, "entropy": r.entropy}
    if s.top:
        out["top_ids"], out["top_logprobs"] = r.top_ids, r.top_logprobs
    return out


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held(x):
    """What pages of 16 tokens (last but two: token, last: dim) hold of x: nearest e4m3 multiples of the page's scale."""
    top = x.abs().amax((-1, -3), keepdim=True)
    e = torch.frexp(top / 448.0)[1]                    # top / 448 in [2^(e-1), 2^e); the smaller one if it is met exactly
    e = torch.where(448.0 * _two_to(e - 1) == top, e - 1, e)
    s = _two_to(torch.where(top > 0, e.clamp(-100, 119), torch.zeros_like(e)))
    y = x / s
    step = _two_to((torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step * s


def _held_sequence(old, new):
    """A sequence's cached values in 64 bits: old rows held first, then the new rows with what shares their first page."""
    def pages(x):
        n = x.shape[0]
        y = torch.cat([x, x.new_zeros((-n % PAGE,) + x.shape[1:])]).reshape(-1, PAGE, *x.shape[1:])
        return _held(y).reshape(-1, *x.shape[1:])[:n]
    old = pages(old.double())
    whole = old.shape[0] - old.shape[0] % PAGE
    return torch.cat([old[:whole], pages(torch.cat([old[whole:], new.double()]))])


def exact(case, seed):
    if case["op"] == "place":
        return None
    if case["op"] == "score":
        logits, tokens = _score_inputs(case, seed)
        parts = {"logprob": [], "entropy": [], "top_logprobs": []}
        for a in range(0, case["rows"], 256):
            x, t = logits[a:a + 256].double(), tokens[a:a + 256].long()
            logp = torch.log_softmax(x, -1)
            parts["logprob"].append(logp.gather(1, t[:, None])[:, 0])
            parts["entropy"].append(-(torch.exp(logp) * logp.clamp(min=-1e30)).sum(-1))
            val = torch.sort(logp, dim=-1, descending=True)[0][:, :case["top"]]
            parts["top_logprobs"].append(torch.nn.functional.pad(val, (0, case["top"] - val.shape[1]), value=-math.inf))
        out = {k: torch.cat(v) for k, v in parts.items()}
        if not case["top"]:
            return {"logprob": out["logprob"], "entropy": out["entropy"]}
        return {"logprob": out["logprob"], "entropy": out["entropy"], "top_ids": None, "top_logprobs": out["top_logprobs"]}
    g, ctx, q, old, new = _kv_inputs(case, seed)
    n_kv = case["n_kv"]
    if case["op"] == "append":
        held = [[], []]
        for i in range(2):
            shared, fresh, a, b = [], [], 0, 0
            for c, k in zip(ctx, q):
                x = _held_sequence(old[i][a:a + c], new[i][b:b + k])
                a, b = a + c, b + k
                if k:
                    shared.append(x[c - c % PAGE:c])
                fresh.append(x[c:])
            held[i] = torch.cat(shared + fresh)
        return held
    n_q = case["n_q"]
    if n_q * sum(k * (c + k) for c, k in zip(ctx, q)) > 2 ** 31:
        return None
    n_blocks = sum((c + PAGE - 1) // PAGE for c in ctx) + sum(q) // PAGE + 2 * case["n_seq"]
    torch.randperm(n_blocks, generator=g, device=DEV)
    queries = torch.randn((sum(q), n_q, HD), generator=g, device=DEV).to(DTYPES[case["dtype"]]).double()
    out, a, b = [], 0, 0
    for c, k in zip(ctx, q):
        kv = [_held_sequence(old[i][a:a + c], new[i][b:b + k]) for i in range(2)]
        seen = torch.arange(c + k, device=DEV)[None] <= c + torch.arange(k, device=DEV)[:, None]
        heads = []
        for h in range(n_q):
            kk, vv = (x[:, h // (n_q // n_kv)] for x in kv)
            sc = (queries[b:b + k, h] @ kk.T / 8.0).masked_fill(~seen, -math.inf)
            heads.append(torch.softmax(sc, -1) @ vv)
        out.append(torch.stack(heads, 1))
        a, b = a + c, b + k
    return torch.cat(out)
