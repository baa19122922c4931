"""Scores of tokens under rows of logits (include/hsd.h: hsd_token_logprobs)."""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.HSD_BF16, torch.float32: B.HSD_FP32}
_SPLIT = 65536     # a row of fewer logits is not split over workgroups and takes no workspace


class TokenScores(NamedTuple):
    logprob: torch.Tensor       # fp32 [rows]: log p(tokens[r]), natural logarithm
    entropy: torch.Tensor       # fp32 [rows], in nats
    top_ids: torch.Tensor       # int32 [rows, n_top], the most probable first, -1 where there is none
    top_logprobs: torch.Tensor  # fp32 [rows, n_top], -inf where there is none


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, n_top: int = 0) -> TokenScores:
    """Log probability of tokens[r] under softmax(logits[r]), the entropy of that distribution and its n_top most probable
    tokens (the lower id first among equals).  logits: [rows, vocab] bfloat16 or float32, rows may lie apart; tokens: int32
    [rows], an id outside the vocabulary has log probability -inf.  A logit of -inf is a probability of 0.  Enqueues on
    torch's current stream of the tensors' device; no gradient."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise ValueError("logits must be a tensor on a GPU; there is no CPU fallback")
    if logits.dtype not in _TYPES:
        raise ValueError(f"logits: bfloat16 or float32, got {logits.dtype}")
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError(f"logits must be [rows, vocab], got {tuple(logits.shape)}")
    n, vocab = logits.shape
    stride = logits.stride(0) if n > 1 else vocab
    if (vocab > 1 and n > 0 and logits.stride(1) != 1) or stride < vocab:
        raise ValueError("logits: a row's values must lie one after the other and rows must not overlap")
    index = logits.get_device()
    if not isinstance(tokens, torch.Tensor) or tokens.get_device() != index or tokens.dtype != torch.int32 or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous int32 tensor on the logits' device")
    if tokens.shape != (n,):
        raise ValueError(f"tokens must be [{n}], got {tuple(tokens.shape)}")
    if not 0 <= n_top <= B.HSD_MAX_TOP:
        raise ValueError(f"n_top must lie in 0 .. {B.HSD_MAX_TOP}, got {n_top}")
    dev = logits.device
    logprob = torch.empty(n, dtype=torch.float32, device=dev)
    entropy = torch.empty(n, dtype=torch.float32, device=dev)
    ids = torch.empty((n, n_top), dtype=torch.int32, device=dev)
    top = torch.empty((n, n_top), dtype=torch.float32, device=dev)
    nb = B.hsd_token_logprobs_bytes(n, vocab, n_top) if vocab >= _SPLIT else 0
    ws = torch.empty(nb, dtype=torch.uint8, device=dev) if nb else None
    with B.on_device(index):
        B.hsd_token_logprobs(B.current_stream(index), n, vocab, _TYPES[logits.dtype], logits.data_ptr(), stride, tokens.data_ptr(),
                             logprob.data_ptr(), entropy.data_ptr(), n_top, ids.data_ptr(), top.data_ptr(), ws.data_ptr() if nb else None, nb)
    return TokenScores(logprob, entropy, ids, top)
