"""GPU: a decoding loop whose draft cache stays within a budget, from its operators together: attention that appends a row and sums
the weights of all rows in place, eviction into the other of two buffers whenever the cache is full, the verdict on the drafted words and
their log probabilities.  Every step is compared with 64-bit arithmetic over the rows that the loop has kept so far; what stays is checked
against the library's own sums, which those are compared with.  Eagerly and from a captured graph, replayed with other inputs."""
import math

import numpy as np
import pytest
import torch

from parity_util import assert_close, host
from test_gpu_attention_mass import reference
from test_gpu_evict import kept_rows

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


class Loop:
    """Two buffers of `room` rows; the cache holds at most that many and is cut to `keep` when it is full."""

    def __init__(self, hippo, dtype, B, H, Hkv, d, ctx, room, keep, first, recent, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.h, self.n, self.room, self.keep, self.first, self.recent = hippo, ctx, room, keep, first, recent
        self.k, self.v = ([torch.zeros((B, Hkv, room, d), dtype=TYPES[dtype], device="cuda") for _ in range(2)] for _ in range(2))
        self.mass = [torch.zeros((B, Hkv, room), device="cuda") for _ in range(2)]
        self.at, self.evictions = 0, 0
        for x in (self.k[0], self.v[0]):
            x[:, :, :ctx] = torch.randn((B, Hkv, ctx, d), generator=g, device="cuda").to(x.dtype)
        self.mass[0][:, :, :ctx] = torch.rand((B, Hkv, ctx), generator=g, device="cuda")

    def step(self, q, k_new, v_new):
        if self.n + q.shape[1] > self.room:
            a, b = self.at, 1 - self.at
            self.idx = self.h.hippo_evict_kv(self.mass[a], self.keep, self.k[a], self.v[a], n_rows=self.n, n_first=self.first,
                                             n_recent=self.recent, k_dst=self.k[b], v_dst=self.v[b], mass_dst=self.mass[b])[0]
            self.at, self.n, self.evictions = b, self.keep, self.evictions + 1
        i = self.at
        call = self.h.hippo_draft_attention_mass if q.shape[1] == 1 else self.h.hippo_verify_attention_mass
        out, mass = call(q, self.k[i], self.v[i], self.mass[i], self.n, mass_out=self.mass[i], k_new=k_new, v_new=v_new)
        assert mass.data_ptr() == self.mass[i].data_ptr()
        self.n += q.shape[1]
        return out


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,d,ctx,room,keep", [(1, 4, 2, 64, 90, 96, 60), (2, 14, 2, 64, 300, 310, 200), (1, 28, 4, 128, 1200, 1210, 1000)])
def test_a_generation_within_a_budget(hippo, dtype, B, H, Hkv, d, ctx, room, keep):
    loop = Loop(hippo, dtype, B, H, Hkv, d, ctx, room, keep, 4, 16, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    k = loop.k[0][:, :, :ctx].clone()                             # the rows that a plain program would hold
    v = loop.v[0][:, :, :ctx].clone()
    mass = loop.mass[0][:, :, :ctx].double()
    slack = torch.zeros_like(mass)                                # what the sums may be off by so far
    for t in range(40):
        n_q = 3 if t % 7 == 6 else 1
        q = (2 * torch.randn((B, n_q, H, d), generator=g, device="cuda")).to(TYPES[dtype])
        k_new, v_new = (torch.randn((B, n_q, Hkv, d), generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
        had = loop.evictions
        own = loop.mass[loop.at][:, :, :loop.n].clone()
        out = loop.step(q, k_new, v_new)
        if loop.evictions > had:
            idx = loop.idx.long()
            np.testing.assert_array_equal(idx.cpu().numpy(), kept_rows(own.cpu().numpy(), keep, 4, 16))
            rows = idx[..., None].expand(*idx.shape, d)
            k, v, mass, slack = torch.gather(k, 2, rows), torch.gather(v, 2, rows), torch.gather(mass, 2, idx), torch.gather(slack, 2, idx)
        k, v = (torch.cat([a, b.transpose(1, 2)], 2) for a, b in ((k, k_new), (v, v_new)))
        n = k.shape[2] - n_q
        assert torch.equal(loop.k[loop.at][:, :, :loop.n], k) and torch.equal(loop.v[loop.at][:, :, :loop.n], v)
        want, total, bound = reference(q, k, v, n, mass, 0)
        assert_close(host(out), want.cpu().numpy(), dtype, "step %d" % t)
        slack = torch.cat([slack, torch.zeros_like(slack[:, :, :n_q])], 2) + bound
        mass = total
        assert bool(((loop.mass[loop.at][:, :, :loop.n].double() - mass).abs() <= slack).all()), t
    assert loop.evictions >= 1


def test_drafted_words_are_judged_and_weighed(hippo):
    # the verdict and the log probabilities read the same rows of logits
    r = np.random.default_rng(4)
    B, gamma, V = 3, 5, 32000
    p = torch.from_numpy(2 * r.standard_normal((B, gamma + 1, V))).to(torch.bfloat16).cuda()
    best = p[:, :gamma].float().argmax(-1).to(torch.int32)
    best[1, 2] = 7                                                # one word that greedy decoding rejects
    n_acc, nxt = hippo.hippo_spec_verify(p, None, best, None, None, 0.0)
    words = torch.cat([best, nxt[:, None]], 1)
    words[torch.arange(gamma + 1, device="cuda")[None] > n_acc[:, None]] = -1       # padding behind each answer's end
    words[torch.arange(B, device="cuda"), n_acc.long()] = nxt
    lp, ent, ids, top = hippo.hippo_token_logprobs(p, words, 1.0, n_top=1)
    assert n_acc.tolist() == [5, 2, 5]
    said = words >= 0
    assert torch.equal(ids[..., 0][said], words[said]) and torch.equal(top[..., 0][said], lp[said])
    assert bool(torch.isinf(lp[~said]).all()) and bool((ent > 0).all())
    want = torch.log_softmax(p.double(), -1)
    # (rows of 32000 words: 8 words a lane at the most 160 additions and roundings of each, of sums near 1e4; see the operator's tests)
    err = (lp.double() - want.gather(2, words.clamp(min=0).long()[..., None])[..., 0]).abs()[said]
    assert bool((err <= 2.0 ** -24 * (160 + 4 * math.log(V) + 4 * 20)).all())


def test_a_captured_step_and_eviction(hippo):
    B, H, Hkv, d, ctx, room, keep = 1, 28, 4, 128, 1500, 1500, 1000
    def make(seed):
        loop = Loop(hippo, "bf16", B, H, Hkv, d, ctx, room, keep, 4, 16, seed)
        g = torch.Generator(device="cuda").manual_seed(seed + 50)
        q = torch.randn((B, 1, H, d), generator=g, device="cuda").to(torch.bfloat16)
        new = [torch.randn((B, 1, Hkv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        return loop, q, new
    want = []
    for s in (1, 2):
        loop, q, new = make(s)
        out = loop.step(q, *new)                                  # evicts, then appends
        want.append((out.clone(), loop.mass[1].clone(), loop.k[1].clone(), loop.v[1].clone()))
    loop, q, new = make(1)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = loop.step(q, *new)
    for s in (2, 1, 2, 1):
        other, q2, new2 = make(s)
        for dst, src in zip((loop.k[0], loop.v[0], loop.mass[0], q, *new), (other.k[0], other.v[0], other.mass[0], q2, *new2)):
            dst.copy_(src)
        for x in (loop.k[1], loop.v[1], loop.mass[1]):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, loop.mass[1], loop.k[1], loop.v[1]), want[s - 1]))
