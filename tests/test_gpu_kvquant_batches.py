"""Calls around the 8-bit cache that come in other shapes than a packed batch that fits: rows behind the last sequence."""
import numpy as np
import pytest
import torch

from test_gpu_kvquant import HD, PAGE, check_attend, cu_of, dev, fill, make_cache, rand_rows

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
