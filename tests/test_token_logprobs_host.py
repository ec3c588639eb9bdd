"""Refusals of hippo_token_logprobs, without a GPU: the library answers before it launches anything."""
import ctypes as C
import re

import pytest
import torch

import paper_2601_08273_amd as h

FAKE = 0x10000


def call(logits=FAKE, dtype=h.DTYPE_BF16, stride=32000, tokens=FAKE, rows=4, vocab=32000, T=1.0, n_top=5, lp=FAKE, ent=FAKE,
         ids=FAKE, top=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return h.load().hippo_token_logprobs(logits, dtype, stride, tokens, rows, vocab, T, n_top, lp, ent, ids, top, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(logits=None), h.ERR_NULL_ARG), (dict(tokens=None), h.ERR_NULL_ARG), (dict(lp=None), h.ERR_NULL_ARG),
    (dict(ent=None), h.ERR_NULL_ARG), (dict(ids=None), h.ERR_NULL_ARG), (dict(top=None), h.ERR_NULL_ARG),
    (dict(ws=None), h.ERR_NULL_ARG),
    (dict(dtype=h.DTYPE_FP8_E4M3), h.ERR_BAD_DTYPE), (dict(dtype=9), h.ERR_BAD_DTYPE),
    (dict(rows=0), h.ERR_BAD_SHAPE), (dict(rows=-1), h.ERR_BAD_SHAPE), (dict(rows=(1 << 22) + 1), h.ERR_BAD_SHAPE),
    (dict(vocab=0), h.ERR_BAD_SHAPE), (dict(vocab=(1 << 20) + 1, stride=1 << 21), h.ERR_BAD_SHAPE),
    (dict(n_top=-1), h.ERR_BAD_SHAPE), (dict(n_top=33), h.ERR_BAD_SHAPE), (dict(vocab=4, n_top=5), h.ERR_BAD_SHAPE),
    (dict(stride=31992), h.ERR_BAD_SHAPE), (dict(stride=-32000), h.ERR_BAD_SHAPE),
    (dict(T=0.0), h.ERR_BAD_SHAPE), (dict(T=-1.0), h.ERR_BAD_SHAPE), (dict(T=float("nan")), h.ERR_BAD_SHAPE),
    (dict(T=float("inf")), h.ERR_BAD_SHAPE), (dict(T=1e-39), h.ERR_BAD_SHAPE),
    (dict(stride=32004), h.ERR_BAD_ALIGN), (dict(logits=FAKE + 8), h.ERR_BAD_ALIGN), (dict(ws=FAKE + 16), h.ERR_BAD_ALIGN),
    (dict(tokens=FAKE + 2), h.ERR_BAD_ALIGN), (dict(ent=FAKE + 1), h.ERR_BAD_ALIGN), (dict(ids=FAKE + 2), h.ERR_BAD_ALIGN),
    (dict(ws_bytes=0), h.ERR_WORKSPACE_TOO_SMALL),
])
def test_arguments_are_checked(bad, status):
    assert call(**bad) == status


def test_workspace_sizes():
    need = h.load().hippo_token_logprobs_workspace_bytes
    assert need(1, 32000, h.DTYPE_BF16, 5) > 0 and need(1, 32000, h.DTYPE_BF16, 0) > 0
    assert need(0, 32000, h.DTYPE_BF16, 5) == 0 and need(1, 32000, 7, 5) == 0 and need(1, 32000, h.DTYPE_F32, 33) == 0
    big = need(6, 152064, h.DTYPE_BF16, 20)
    assert call(rows=6, vocab=152064, stride=152064, n_top=20, ws_bytes=big - 1) == h.ERR_WORKSPACE_TOO_SMALL


def test_the_binding_refuses_tensors_it_would_misread():
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    for logits, tokens, more in (
            (x.t(), t, {}), (x, t.long(), {}), (x, t[:3], {}), (x, t.view(2, 2), {}), (x[0], t[0], {}),
            (torch.zeros(2, 3, 64)[:, ::2], torch.zeros(2, 2, dtype=torch.int32), {}),      # rows not evenly spaced
            (x, t, dict(logprob_out=torch.zeros(3))), (x, t, dict(entropy_out=torch.zeros(4, dtype=torch.float64))),
            (x, t, dict(n_top=2, top_ids_out=torch.zeros(4, 2))),
            (x, t, dict(n_top=2, top_logprobs_out=torch.zeros(2, 4).t())), (x, t, dict(n_top=-1))):
        with pytest.raises(AssertionError):
            h.hippo_token_logprobs(logits, tokens, **more)
    with pytest.raises(AssertionError):                           # host memory, which no kernel reads
        h.hippo_token_logprobs(x, t)
    with pytest.raises(TypeError):
        h.hippo_token_logprobs(x.double(), t)


@pytest.mark.parametrize("case,part", [
    (dict(x=torch.zeros(64, 4).t()), "x.stride(-1) == 1"), (dict(x=torch.zeros(64)), "x.dim() >= 2"),
    (dict(x=torch.zeros(2, 3, 64)[:, ::2], tokens=torch.zeros(2, 2, dtype=torch.int32)), "x.stride(i) == inside * step"),
    (dict(x=torch.zeros(3, 2, 64).transpose(0, 1), tokens=torch.zeros(2, 3, dtype=torch.int32)), "x.stride(i) == inside * step"),
    (dict(tokens=torch.zeros(4, dtype=torch.int64)), "tokens.scalar_type() == at::kInt"),
    (dict(tokens=torch.zeros(3, dtype=torch.int32)), "tokens.sizes() =="), (dict(tokens=torch.zeros(2, 2, dtype=torch.int32)), "tokens.sizes() =="),
    (dict(tokens=torch.zeros(8, dtype=torch.int32)[::2]), "tokens.is_contiguous()"),
    (dict(logprob_out=torch.zeros(3)), "t.sizes() == sizes"), (dict(logprob_out=torch.zeros(8)[::2]), "t.is_contiguous()"),
    (dict(entropy_out=torch.zeros(4, dtype=torch.float64)), "t.scalar_type() == type"), (dict(entropy_out=torch.zeros(4, 1)), "t.sizes() == sizes"),
    (dict(n_top=2, top_ids_out=torch.zeros(4, 2)), "t.scalar_type() == type"),
    (dict(n_top=2, top_ids_out=torch.zeros(4, 3, dtype=torch.int32)), "t.sizes() == sizes"),
    (dict(n_top=2, top_logprobs_out=torch.zeros(2, 4).t()), "t.is_contiguous()"), (dict(n_top=-1), "n_top >= 0"),
    (dict(), "tensors lie on the current device"),                # nothing else: host memory, which no kernel reads
])
def test_the_binding_names_what_it_refuses(case, part):
    """(all of these tensors lie in host memory, which the last check refuses: each case has to fail at its own check, before it)"""
    case = dict(case)
    with pytest.raises(AssertionError, match=re.escape(part)):
        h.hippo_token_logprobs(case.pop("x", torch.zeros(4, 64)), case.pop("tokens", torch.zeros(4, dtype=torch.int32)), **case)
