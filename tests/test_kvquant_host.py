"""The operators without a context refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

import paper_2602_12957_amd.binding as B

FAKE = 0x10000   # never dereferenced: every call below is refused first


def _kv(**kw):
    kv = B.hsd_kv_quant(FAKE, FAKE, FAKE, FAKE, 64, 4)
    for k, v in kw.items():
        setattr(kv, k, v)
    return kv


def _rows(**kw):
    b = B.hsd_batch()
    b.n_seq, b.total_q, b.max_blocks_per_seq, b.n_slots = 4, 40, 32, 4
    for name in ("cu_q", "seq_len", "block_table", "status"):
        setattr(b, name, FAKE)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


ROWS = [(dict(n_seq=0), B.HSD_EINVAL), (dict(total_q=-1), B.HSD_EINVAL), (dict(max_blocks_per_seq=0), B.HSD_EINVAL),
        (dict(n_slots=0), B.HSD_EINVAL), (dict(n_slots=3), B.HSD_EINVAL), (dict(cu_q=None), B.HSD_EINVAL), (dict(seq_len=None), B.HSD_EINVAL),
        (dict(block_table=None), B.HSD_EINVAL), (dict(tree_end=FAKE), B.HSD_EINVAL), (dict(n_seq=5000, n_slots=5000), B.HSD_ERANGE),
        (dict(max_blocks_per_seq=1 << 28), B.HSD_ERANGE)]
PAGES = [(dict(k_codes=None), B.HSD_EINVAL), (dict(v_codes=None), B.HSD_EINVAL), (dict(k_scale=None), B.HSD_EINVAL),
         (dict(v_scale=None), B.HSD_EINVAL), (dict(n_blocks=0), B.HSD_EINVAL), (dict(n_kv_heads=0), B.HSD_EINVAL),
         (dict(k_codes=FAKE + 8), B.HSD_EINVAL), (dict(v_codes=FAKE + 1), B.HSD_EINVAL), (dict(n_kv_heads=2000), B.HSD_ERANGE),
         (dict(n_blocks=1 << 28), B.HSD_ERANGE)]


def _pool(**kw):
    p = B.hsd_kv_pool(None, None, 64, FAKE, FAKE)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", ROWS)
def test_rows_are_checked(kw, code):
    b, p, kv = _rows(**kw), _pool(), _kv()
    assert B.lib.hsd_kv_reserve(None, C.byref(p), C.byref(b), FAKE, FAKE) == code
    assert B.lib.hsd_kv_commit_rows(None, C.byref(p), C.byref(b)) == code
    assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(b), 16, B.HSD_BF16, 0.125, FAKE, 1024, FAKE, 1024, FAKE, 1 << 30) == code
    assert B.hsd_kv_quant_attention_bytes(kv, b, 16) == 0


@pytest.mark.parametrize("kw,code", PAGES)
def test_pages_are_checked(kw, code):
    b, kv = _rows(), _kv(**kw)
    args = (FAKE, B.HSD_BF16, FAKE, FAKE, 1 << 20, 1 << 20)
    assert B.lib.hsd_kv_quant_append(None, C.byref(kv), 8, *args, FAKE) == code
    assert B.lib.hsd_kv_quant_read(None, C.byref(kv), 8, *args) == code
    assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(b), 16000, B.HSD_BF16, 0.125, FAKE, 1 << 20, FAKE, 1 << 20, FAKE, 1 << 30) == code


def test_reserve_arguments():
    b, p = _rows(), _pool()
    assert B.lib.hsd_kv_reserve(None, None, C.byref(b), FAKE, FAKE) == B.HSD_EINVAL
    assert B.lib.hsd_kv_reserve(None, C.byref(p), None, FAKE, FAKE) == B.HSD_EINVAL
    assert B.lib.hsd_kv_reserve(None, C.byref(p), C.byref(b), None, FAKE) == B.HSD_EINVAL
    assert B.lib.hsd_kv_reserve(None, C.byref(p), C.byref(_rows(status=None)), FAKE, FAKE) == B.HSD_EINVAL
    for kw in (dict(n_blocks=0), dict(free_list=None), dict(free_count=None)):
        assert B.lib.hsd_kv_reserve(None, C.byref(_pool(**kw)), C.byref(b), FAKE, FAKE) == B.HSD_EINVAL
        assert B.lib.hsd_kv_commit_rows(None, C.byref(_pool(**kw)), C.byref(b)) == B.HSD_EINVAL


def test_append_and_read_arguments():
    kv = _kv()
    ok = dict(n=8, slot=FAKE, dtype=B.HSD_BF16, k=FAKE, v=FAKE, ks=256, vs=256)
    for kw in (dict(n=-1), dict(slot=None), dict(dtype=5), dict(k=None), dict(v=None), dict(ks=255), dict(vs=0)):
        a = {**ok, **kw}
        args = (a["n"], a["slot"], a["dtype"], a["k"], a["v"], a["ks"], a["vs"])
        assert B.lib.hsd_kv_quant_append(None, C.byref(kv), *args, None) == B.HSD_EINVAL
        assert B.lib.hsd_kv_quant_read(None, C.byref(kv), *args) == B.HSD_EINVAL
    # no rows: nothing to do, nothing looked at
    assert B.lib.hsd_kv_quant_append(None, C.byref(kv), 0, None, B.HSD_FP32, None, None, 0, 0, None) == B.HSD_OK
    assert B.lib.hsd_kv_quant_read(None, C.byref(kv), 0, None, B.HSD_FP32, None, None, 0, 0) == B.HSD_OK


def test_attention_arguments():
    b, kv = _rows(max_blocks_per_seq=4096), _kv()     # long tables: the keys are split over workgroups, which takes a workspace
    need = B.hsd_kv_quant_attention_bytes(kv, b, 16)
    assert need > 0
    ok = dict(heads=16, dtype=B.HSD_BF16, scale=0.125, q=FAKE, qs=1024, o=FAKE, os=1024, ws=FAKE, nb=need)
    for kw, code in ((dict(heads=0), B.HSD_EINVAL), (dict(heads=18), B.HSD_EINVAL), (dict(dtype=2), B.HSD_EINVAL), (dict(scale=float("nan")), B.HSD_EINVAL),
                     (dict(scale=float("inf")), B.HSD_EINVAL), (dict(q=None), B.HSD_EINVAL), (dict(o=None), B.HSD_EINVAL), (dict(qs=1023), B.HSD_EINVAL),
                     (dict(os=0), B.HSD_EINVAL), (dict(ws=None), B.HSD_EINVAL), (dict(nb=need - 1), B.HSD_ENOSPC),
                     (dict(heads=1028, qs=1 << 20, os=1 << 20), B.HSD_ERANGE), (dict(ws=FAKE + 16), B.HSD_EINVAL)):
        a = {**ok, **kw}
        assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(b), a["heads"], a["dtype"], a["scale"], a["q"], a["qs"], a["o"], a["os"],
                                            a["ws"], a["nb"]) == code
    assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(_rows(total_q=0)), 16, B.HSD_BF16, 0.125, None, 0, None, 0, None, 0) == B.HSD_OK


def test_token_logprobs_arguments():
    need = B.hsd_token_logprobs_bytes(4, 200000, 5)
    assert need > 0 and B.hsd_token_logprobs_bytes(4, 0, 5) == 0 and B.hsd_token_logprobs_bytes(4, 10, 33) == 0 and B.hsd_token_logprobs_bytes(-1, 10, 3) == 0
    ok = dict(n=4, vocab=200000, dtype=B.HSD_FP32, x=FAKE, stride=200000, tok=FAKE, lp=FAKE, ent=FAKE, top=5, ids=FAKE, tlp=FAKE, ws=FAKE, nb=need)
    for kw, code in ((dict(n=-1), B.HSD_EINVAL), (dict(vocab=0), B.HSD_EINVAL), (dict(dtype=9), B.HSD_EINVAL), (dict(x=None), B.HSD_EINVAL),
                     (dict(stride=199999), B.HSD_EINVAL), (dict(tok=None), B.HSD_EINVAL), (dict(lp=None), B.HSD_EINVAL), (dict(ent=None), B.HSD_EINVAL),
                     (dict(top=-1), B.HSD_EINVAL), (dict(top=33), B.HSD_ERANGE), (dict(ids=None), B.HSD_EINVAL), (dict(tlp=None), B.HSD_EINVAL),
                     (dict(ws=None), B.HSD_EINVAL), (dict(nb=need - 1), B.HSD_ENOSPC), (dict(ws=FAKE + 64), B.HSD_EINVAL)):
        a = {**ok, **kw}
        assert B.lib.hsd_token_logprobs(None, a["n"], a["vocab"], a["dtype"], a["x"], a["stride"], a["tok"], a["lp"], a["ent"], a["top"], a["ids"],
                                        a["tlp"], a["ws"], a["nb"]) == code
    assert B.lib.hsd_token_logprobs(None, 0, 1000, B.HSD_FP32, None, 1000, None, None, None, 0, None, None, None, 0) == B.HSD_OK


def test_launches_that_would_not_fit_are_refused():
    kv, big = _kv(), 1 << 60
    assert B.lib.hsd_kv_quant_append(None, C.byref(kv), (1 << 29) + 1, FAKE, B.HSD_BF16, FAKE, FAKE, big, big, None) == B.HSD_ERANGE
    assert B.lib.hsd_kv_quant_read(None, C.byref(kv), (1 << 29) + 1, FAKE, B.HSD_FP32, FAKE, FAKE, big, big) == B.HSD_ERANGE
    b = _rows(total_q=(1 << 25) + 1)
    assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(b), 16, B.HSD_BF16, 0.125, FAKE, 1024, FAKE, 1024, FAKE, 1 << 40) == B.HSD_ERANGE
    # a scale that is finite, but not in powers of two
    assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(_rows()), 16, B.HSD_BF16, 3e38, FAKE, 1024, FAKE, 1024, None, 0) == B.HSD_EINVAL
    assert B.lib.hsd_token_logprobs(None, 1 << 24, 8, B.HSD_FP32, FAKE, 8, FAKE, FAKE, FAKE, 0, None, None, None, 0) == B.HSD_ERANGE
    # decoder passes: no context, no pages
    for fn in (B.lib.hsd_verify_quant, B.lib.hsd_prefill_quant):
        assert fn(None, None, C.byref(_pool()), C.byref(kv), C.byref(_rows()), FAKE, 1 << 40) == B.HSD_EINVAL
    assert B.hsd_workspace_quant_bytes(B.hsd_model_desc(), 16, 1, 8) == 0


def test_without_a_gpu_there_is_no_fallback():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2602_12957_amd.kvquant import QuantKV
    from paper_2602_12957_amd.scoring import token_logprobs
    with pytest.raises(RuntimeError):
        QuantKV(4, 1, 1, 4)
    with pytest.raises(ValueError):
        QuantKV(0, 1, 1, 4)
    with pytest.raises(ValueError):
        token_logprobs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32))


def test_rows_and_positions_whose_sums_pass_32_bits_are_refused():
    """As many rows as append and read take, and tables whose positions leave room for them in 31 bits."""
    kv, p = _kv(), _pool()
    widest = ((1 << 31) - 1 - (1 << 29)) // 16
    for kw in (dict(total_q=(1 << 29) + 1), dict(total_q=(1 << 31) - 1), dict(max_blocks_per_seq=widest + 1)):
        b = _rows(**kw)
        assert B.lib.hsd_kv_reserve(None, C.byref(p), C.byref(b), FAKE, FAKE) == B.HSD_ERANGE
        assert B.lib.hsd_kv_commit_rows(None, C.byref(p), C.byref(b)) == B.HSD_ERANGE
        assert B.lib.hsd_kv_quant_attention(None, C.byref(kv), C.byref(b), 16, B.HSD_BF16, 0.125, FAKE, 1024, FAKE, 1024, FAKE, 1 << 40) == B.HSD_ERANGE
        assert B.hsd_kv_quant_attention_bytes(kv, b, 16) == 0
    assert B.hsd_kv_quant_attention_bytes(kv, _rows(max_blocks_per_seq=widest), 16) > 0


def test_a_decoder_of_trees_is_refused_on_an_8bit_cache():
    from types import SimpleNamespace

    from paper_2602_12957_amd.specdecode import SpecDecoder
    with pytest.raises(ValueError, match="packed trees"):
        SpecDecoder(SimpleNamespace(layers8=(B.hsd_kv_quant * 1)()))
    assert SpecDecoder(SimpleNamespace(layers8=None)).mode == "region"
