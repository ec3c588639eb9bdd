"""Refusals of hippo_*_attention_mass, without a GPU: the library answers before it launches anything."""
import ctypes as C
import re

import pytest
import torch

import paper_2601_08273_amd as h

FAKE = 0x10000


def desc(rows=20000, **more):
    d = dict(batch=2, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=h.DTYPE_BF16)
    d.update(more)
    d.setdefault("stride_n", d["head_dim"])
    d.setdefault("stride_h", rows * d["head_dim"])
    d.setdefault("stride_b", d["n_kv_heads"] * rows * d["head_dim"])
    return h.KvDesc(**d)


def call(fn, q=FAKE, q_len=6, k_new=None, v_new=None, k=FAKE, v=2 * FAKE, kv=None, ctx=16640, splits=0, out=FAKE, m_in=FAKE,
         m_out=3 * FAKE, isb=80000, ish=20000, osb=80000, osh=20000, ws=FAKE, ws_bytes=1 << 40, no_kv=False, no_mass=False):
    mass = None if no_mass else C.byref(h.MassDesc(m_in, m_out, isb, ish, osb, osh))
    return fn(q, q_len, k_new, v_new, k, v, None if no_kv else C.byref(kv or desc()), ctx, 0.0, splits, out, None, mass, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(no_kv=True), h.ERR_NULL_ARG), (dict(no_mass=True), h.ERR_NULL_ARG), (dict(m_out=None), h.ERR_NULL_ARG),
    (dict(q=None), h.ERR_NULL_ARG), (dict(k=None), h.ERR_NULL_ARG), (dict(v=None), h.ERR_NULL_ARG), (dict(out=None), h.ERR_NULL_ARG),
    (dict(ws=None), h.ERR_NULL_ARG), (dict(k_new=FAKE), h.ERR_NULL_ARG), (dict(v_new=FAKE), h.ERR_NULL_ARG),
    (dict(osh=16645), h.ERR_BAD_SHAPE), (dict(osb=0), h.ERR_BAD_SHAPE), (dict(ish=-1), h.ERR_BAD_SHAPE),
    (dict(m_in=3 * FAKE, ish=19999), h.ERR_BAD_SHAPE), (dict(m_in=3 * FAKE, isb=1), h.ERR_BAD_SHAPE),
    (dict(q_len=0), h.ERR_BAD_SHAPE), (dict(ctx=-1), h.ERR_BAD_SHAPE), (dict(splits=-1), h.ERR_BAD_SHAPE), (dict(q_len=600), h.ERR_BAD_SHAPE),
    (dict(kv=desc(dtype=h.DTYPE_FP8_E4M3)), h.ERR_BAD_DTYPE), (dict(kv=desc(dtype=7)), h.ERR_BAD_DTYPE),
    (dict(kv=desc(head_dim=96)), h.ERR_BAD_SHAPE), (dict(kv=desc(n_q_heads=27)), h.ERR_BAD_SHAPE),
    (dict(m_in=FAKE + 2), h.ERR_BAD_ALIGN), (dict(m_out=3 * FAKE + 1), h.ERR_BAD_ALIGN), (dict(k=FAKE + 8), h.ERR_BAD_ALIGN),
    (dict(k_new=FAKE + 8, v_new=FAKE), h.ERR_BAD_ALIGN), (dict(ws=FAKE + 128), h.ERR_BAD_ALIGN),
    (dict(ws_bytes=1 << 20), h.ERR_WORKSPACE_TOO_SMALL),
])
def test_arguments_are_checked(bad, status):
    for fn in (h.load().hippo_verify_attention_mass, h.load().hippo_draft_attention_mass):
        assert call(fn, **bad) == status


def test_workspace_sizes():
    need = h.load().hippo_attention_mass_workspace_bytes
    kv = desc()
    n = need(C.byref(kv), 6, 16646, 0)
    assert n > h.workspace_bytes(h.CALL_VERIFY_ATTENTION, kv, None, 6, 16646)
    assert call(h.load().hippo_verify_attention_mass, ws_bytes=n - 1) == h.ERR_WORKSPACE_TOO_SMALL
    assert need(C.byref(desc(dtype=h.DTYPE_FP8_E4M3)), 6, 16646, 0) == 0 and need(None, 6, 16646, 0) == 0
    assert need(C.byref(kv), 6, 5, 0) == 0 and need(C.byref(kv), 0, 5, 0) == 0


def test_the_binding_refuses_tensors_it_would_misread():
    q, k, v, m = torch.zeros(2, 2, 6, 64), torch.zeros(2, 3, 50, 64), torch.zeros(2, 3, 50, 64), torch.zeros(2, 3, 48)
    for args, more in (
            ((q, k, v, m.double(), 48), {}), ((q, k, v, m[:1], 48), {}), ((q, k, v, m[:, :, :47], 48), {}), ((q, k, v, m, 49), {}),
            ((q, k, v, m, -1), {}), ((q.bfloat16(), k, v, m, 48), {}), ((q[:1], k, v, m, 48), {}), ((q, k, v.bfloat16(), m, 48), {}),
            ((q, k, v.transpose(1, 2).contiguous().transpose(1, 2), m, 48), {}), ((q.transpose(0, 1), k, v, m, 48), {}),
            ((q, k, v, m.transpose(1, 2).contiguous().transpose(1, 2), 48), {}),
            ((q, k, v, m, 48), dict(mass_out=torch.zeros(2, 3, 49))), ((q, k, v, m, 48), dict(mass_out=torch.zeros(2, 3, 50).double())),
            ((q, k, v, m, 48), dict(out=torch.zeros(2, 2, 6, 32))), ((q, k, v, m, 48), dict(out=q.bfloat16())),
            ((q, k, v, m, 48), dict(k_new=torch.zeros(2, 2, 3, 64))),
            ((q, k, v, m, 48), dict(k_new=torch.zeros(2, 1, 3, 64), v_new=torch.zeros(2, 2, 3, 64))),
            ((q, k, v, m, 48), {})):                               # host memory, which no kernel reads
        with pytest.raises(AssertionError):
            h.hippo_verify_attention_mass(*args, **more)


@pytest.mark.parametrize("strides,status", [
    (dict(osb=20000, osh=20000), h.ERR_BAD_SHAPE),                 # head 1 of the first sequence on head 0 of the second
    (dict(osb=76645, osh=20000), h.ERR_BAD_SHAPE), (dict(osb=76646, osh=20000), h.ERR_WORKSPACE_TOO_SMALL),
    (dict(osb=16646, osh=33291), h.ERR_BAD_SHAPE), (dict(osb=16646, osh=33292), h.ERR_WORKSPACE_TOO_SMALL),
    (dict(osb=40000, osh=20000), h.ERR_BAD_SHAPE), (dict(osb=17000, osh=50000), h.ERR_WORKSPACE_TOO_SMALL),
    (dict(osb=0, osh=0), h.ERR_BAD_SHAPE), (dict(isb=0, ish=0), h.ERR_WORKSPACE_TOO_SMALL),          # `in` is only read
    (dict(m_in=3 * FAKE, isb=20000, ish=20000, osb=20000, osh=20000), h.ERR_BAD_SHAPE),              # in place
    (dict(kv=desc(batch=1), osb=0), h.ERR_WORKSPACE_TOO_SMALL), (dict(kv=desc(n_kv_heads=1), osh=0), h.ERR_WORKSPACE_TOO_SMALL),
])
def test_rows_of_mass_that_would_meet_are_refused(strides, status):
    for fn in (h.load().hippo_verify_attention_mass, h.load().hippo_draft_attention_mass):
        assert call(fn, ws_bytes=256, **strides) == status


@pytest.mark.parametrize("case,part", [
    (dict(mass=lambda m: m.double()), "mass.scalar_type() == at::kFloat"), (dict(mass=lambda m: m[0]), "mass.dim() == 3"),
    (dict(mass=lambda m: m[:1]), "mass.size(0) == B"), (dict(mass=lambda m: m[:, :2]), "mass.size(1) == Hkv"),
    (dict(mass=lambda m: m[:, :, :47]), "mass.size(2) >= n"),
    (dict(mass=lambda m: m.transpose(1, 2).contiguous().transpose(1, 2)), "mass.stride(2) == 1"),
    (dict(ctx=49), "n <= k.size(2)"), (dict(ctx=-1), "c.ctx_len >= 0"),
    (dict(q=lambda q: q.bfloat16()), "c.q.scalar_type() == k.scalar_type()"), (dict(q=lambda q: q[:1]), "c.q.size(0) == B"),
    (dict(q=lambda q: q[:, :0]), "c.q.size(1) >= 1"), (dict(q=lambda q: q[..., :32].contiguous()), "c.q.size(3) == k.size(3)"),
    (dict(q=lambda q: q.transpose(0, 1)), "q.is_contiguous()"), (dict(q=lambda q: q[0]), "q.dim() == 4"),
    (dict(k=lambda k: k[..., ::2]), "cache.stride(3) == 1"), (dict(k=lambda k: k[0]), "cache.dim() == 4"),
    (dict(v=lambda v: v.bfloat16()), "v.scalar_type() == k.scalar_type()"),
    (dict(v=lambda v: v.transpose(1, 2).contiguous().transpose(1, 2)), "same_layout(v, k)"), (dict(v=lambda v: v[:, :, :49]), "same_layout(v, k)"),
    (dict(mass_out=torch.zeros(2, 3, 49)), "mass.size(2) >= n"), (dict(mass_out=torch.zeros(2, 3, 50).double()), "mass.scalar_type() == at::kFloat"),
    (dict(mass_out=torch.zeros(2, 50, 3).transpose(1, 2)), "mass.stride(2) == 1"),
    (dict(out=torch.zeros(2, 2, 6, 32)), "t.sizes() == sizes"), (dict(out=torch.zeros(2, 2, 6, 64).bfloat16()), "t.scalar_type() == type"),
    (dict(out=torch.zeros(2, 6, 2, 64).transpose(1, 2)), "t.is_contiguous()"),
    (dict(k_new=torch.zeros(2, 2, 3, 64)), "k_new.defined() == v_new.defined()"),
    (dict(v_new=torch.zeros(2, 2, 3, 64)), "k_new.defined() == v_new.defined()"),
    (dict(k_new=torch.zeros(2, 1, 3, 64), v_new=torch.zeros(2, 2, 3, 64)), "t->sizes()"),
    (dict(k_new=torch.zeros(2, 2, 3, 64), v_new=torch.zeros(2, 2, 2, 64)), "t->sizes()"),
    (dict(k_new=torch.zeros(2, 2, 3, 64), v_new=torch.zeros(2, 3, 2, 64).transpose(1, 2)), "t->is_contiguous()"),
    (dict(k_new=torch.zeros(2, 2, 3, 64), v_new=torch.zeros(2, 2, 3, 64).bfloat16()), "t->scalar_type() == k.scalar_type()"),
    (dict(), "tensors lie on the current device"),                # nothing else: host memory, which no kernel reads
])
@pytest.mark.parametrize("fn", [h.hippo_draft_attention_mass, h.hippo_verify_attention_mass])
def test_the_binding_names_what_it_refuses(fn, case, part):
    """(all of these tensors lie in host memory, which the last check refuses: each case has to fail at its own check, before it)"""
    case = dict(case)
    q, k, v, m = torch.zeros(2, 2, 6, 64), torch.zeros(2, 3, 50, 64), torch.zeros(2, 3, 50, 64), torch.zeros(2, 3, 48)
    q, k, v, m = (case.pop(name, lambda x: x)(x) for name, x in (("q", q), ("k", k), ("v", v), ("mass", m)))
    with pytest.raises(AssertionError, match=re.escape(part)):
        fn(q, k, v, m, case.pop("ctx", 48), **case)
