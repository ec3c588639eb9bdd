"""A draft cache that stays within a budget while an answer grows, and what the answer's words were worth.

A long answer lets the draft model's cache grow past what its compute pays for.  Three operators bound it and report on it:

  mass      attention of the newest rows over a cache that also adds up, for every cache row and KV head, how much weight the
            query heads gave it (hippo_draft_attention_mass for single tokens, hippo_verify_attention_mass for several)
  evict     a new cache of the rows worth keeping by that weight: the first rows, the most recent ones, and of those between
            the ones with the most accumulated weight, chosen for each KV head by itself (hippo_evict_kv)
  logprobs  log probabilities of an answer's words under the model's logits, with the distribution's entropy and its most
            likely words (hippo_token_logprobs)

Head layouts and cache lengths are those of synth_inputs.py's configurations (832, 16K, 33K and 4 x 37K rows, and the draft
caches that pruning leaves of them); `draw` gives ragged ones around them.

`own` False computes the operators in elementary torch operations, True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head dim) of the configurations
HEADS = {"4/2x64": (4, 2, 64), "14/2x64": (14, 2, 64), "28/4x128": (28, 4, 128), "64/8x128": (64, 8, 128)}
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}
ELEM_BYTES = {"fp32": 4, "bf16": 2, "fp8": 1}


def _mass(name, dtype, batch, heads, ctx, q_len, append):
    return dict(name=name, op="mass", dtype=dtype, batch=batch, heads=heads, ctx=ctx, q_len=q_len, append=append)


def _evict(name, dtype, batch, heads, rows, keep, first, recent):
    return dict(name=name, op="evict", dtype=dtype, batch=batch, heads=heads, rows=rows, keep=keep, first=first, recent=recent)


def _logprobs(name, dtype, rows, vocab, top, temperature):
    return dict(name=name, op="logprobs", dtype=dtype, rows=rows, vocab=vocab, top=top, temperature=temperature)


def listed():
    return [
        # the smallest call: one token over a short fp32 cache (latency and launches)
        _mass("mass_fp32_832", "fp32", 1, "4/2x64", 832, 1, False),
        # a decoding step of the draft model over the cache that pruning left of 16K visual tokens: the call that a generation
        # makes most often, its row appended by the call
        _mass("mass_draft_1.9k", "bf16", 1, "28/4x128", 1895, 1, True),
        # a decoding step over a cache that is not pruned yet
        _mass("mass_16k", "bf16", 1, "28/4x128", 16640, 1, False),
        # a chain of five draft tokens verified over the same cache
        _mass("mass_verify_16k", "bf16", 1, "28/4x128", 16640, 6, True),
        # a decoding step of a batch of a large model: the most bytes
        _mass("mass_4x37k", "bf16", 4, "64/8x128", 37120, 1, False),
        # eviction from a short fp32 cache: launches
        _evict("evict_fp32_832", "fp32", 1, "14/2x64", 832, 416, 4, 64),
        # the ordinary one: half of an unpruned cache goes
        _evict("evict_16k", "bf16", 1, "28/4x128", 16657, 8192, 4, 256),
        # a long video's cache in 8 bits, of which a tenth stays
        _evict("evict_fp8_33k", "fp8", 1, "28/4x128", 33280, 3328, 0, 128),
        # a batch of a large model: the most bytes
        _evict("evict_4x37k", "bf16", 4, "64/8x128", 37133, 12288, 16, 1024),
        # the word just drawn, with its five best alternatives, beside a decoding step
        _logprobs("logprobs_1x32000", "fp32", 1, 32000, 5, 1.0),
        # a verified chain's rows
        _logprobs("logprobs_6x152k", "bf16", 6, 152064, 20, 1.0),
        # whole answers scored at once: a batch's words, no alternatives but the best one
        _logprobs("logprobs_1000x152k", "bf16", 1000, 152064, 1, 0.7),
    ]


# ---------------------------------------------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(["mass", "mass", "evict", "logprobs"])
    if op == "logprobs":
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp32"]), rows=_log_int(rng, 1, 1000),
                    vocab=_log_int(rng, 1000, 160000), top=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]),
                    temperature=rng.choice([1.0, 1.0, 0.7, 1.3]))
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp32"]), batch=rng.choice([1, 1, 2, 3, 4]), heads=rng.choice(sorted(HEADS)))
    if op == "mass":
        case.update(ctx=_log_int(rng, 64, 37120), q_len=rng.choice([1, 1, 1, rng.randint(2, 9)]), append=rng.random() < 0.5)
    else:
        rows = _log_int(rng, 256, 40000)
        first, recent = rng.choice([0, 4, 16]), rng.randint(1, rows // 16)
        case.update(dtype=rng.choice([case["dtype"], "fp8"]), rows=rows, first=first, recent=recent,
                    keep=rng.randint(first + recent + 1, max(rows // 2, first + recent + 1)))
    return case


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e14


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("mass", "evict", "logprobs")}
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most[case["op"]]:
            return case


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _attention_inputs(case, g):
    """Caches whose rows matter differently: of every KV head one row in fifty lies along the direction that its queries
    share, as the tokens that attention keeps coming back to do."""
    H, Hkv, d = HEADS[case["heads"]]
    B, n_q = case["batch"], case["q_len"]
    n, t = case["ctx"] + n_q, TORCH_DTYPE[case["dtype"]]
    shared = torch.nn.functional.normalize(_normal(g, B, Hkv, 1, d), dim=-1)
    k, v = (torch.empty((B, Hkv, n, d), dtype=t, device="cuda") for _ in range(2))
    for b in range(B):
        heavy = (torch.rand((Hkv, n, 1), generator=g, device="cuda") < 0.02).float()
        k[b] = _normal(g, Hkv, n, d) + 4.0 * heavy * shared[b]
        v[b] = _normal(g, Hkv, n, d)
    q = _normal(g, B, n_q, Hkv, H // Hkv, d) + 0.6 * math.sqrt(d) * shared.view(B, 1, Hkv, 1, d)
    s = dict(q=q.reshape(B, n_q, H, d).to(t), k=k, v=v, k_new=None, v_new=None)
    if case["append"]:
        s["k_new"], s["v_new"] = (x[:, :, case["ctx"]:].transpose(1, 2).contiguous() for x in (k, v))
    s["mass"] = _accumulated(g, B, Hkv, case["ctx"])
    return s


def _accumulated(g, B, Hkv, n):
    """What the first steps left: a few heavy rows, a long tail, rows that no head has looked at."""
    mass = torch.exp(2.0 * _normal(g, B, Hkv, n)) * (2.0 / n)
    return mass * (torch.rand((B, Hkv, n), generator=g, device="cuda") > 0.05)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "mass":
        return dict(case=case, **_attention_inputs(case, g))
    if case["op"] == "evict":
        H, Hkv, d = HEADS[case["heads"]]
        B, n, t = case["batch"], case["rows"], TORCH_DTYPE[case["dtype"]]
        s = dict(case=case, mass=_accumulated(g, B, Hkv, n))
        for name in ("k", "v"):
            if case["dtype"] == "fp8":     # E4M3 codes: any byte
                s[name] = torch.randint(0, 256, (B, Hkv, n, d), generator=g, device="cuda", dtype=t)
            else:
                s[name] = torch.stack([_normal(g, Hkv, n, d).to(t) for _ in range(B)])
        return s
    # rows of an LM head: a few likely words above a long tail, some words masked; rows 16-byte aligned, as a padded head's are
    R, V, t = case["rows"], case["vocab"], TORCH_DTYPE[case["dtype"]]
    x = torch.empty((R, (V + 7) // 8 * 8), dtype=t, device="cuda")[:, :V]
    tokens = torch.empty((R,), dtype=torch.int32, device="cuda")
    for r0 in range(0, R, 250):
        n = min(250, R - r0)
        y = _normal(g, n, V).mul_(2.0)
        hot = torch.randint(0, V, (n, 4), generator=g, device="cuda")
        y.scatter_reduce_(1, hot, y.max() + 4.0 * torch.rand((n, 4), generator=g, device="cuda"), "amax")
        y.masked_fill_(torch.rand((n, V), generator=g, device="cuda") < 0.01, -math.inf)
        x[r0:r0 + n] = y.to(t)
        tail = torch.randint(0, V, (n,), generator=g, device="cuda")
        tokens[r0:r0 + n] = torch.where(torch.rand((n,), generator=g, device="cuda") < 0.8, hot[:, 0], tail).to(torch.int32)
    return dict(case=case, logits=x, tokens=tokens)


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _call(s):
    """The pass as the library's user writes it."""
    import paper_2601_08273_amd as h
    case = s["case"]
    if case["op"] == "mass":
        attention = h.hippo_draft_attention_mass if case["q_len"] == 1 else h.hippo_verify_attention_mass
        out, mass = attention(s["q"], s["k"], s["v"], s["mass"], case["ctx"], k_new=s["k_new"], v_new=s["v_new"])
        return dict(out=out, mass=mass, k_new=s["k"][:, :, case["ctx"]:], v_new=s["v"][:, :, case["ctx"]:])
    if case["op"] == "evict":
        idx, k, v, mass = h.hippo_evict_kv(s["mass"], case["keep"], s["k"], s["v"], n_first=case["first"],
                                           n_recent=case["recent"])
        return dict(idx=idx, k=k, v=v, mass=mass)
    got = h.hippo_token_logprobs(s["logits"], s["tokens"], case["temperature"], n_top=case["top"])
    return dict(zip(("logprob", "entropy", "top_ids", "top_logprobs"), got))


def _plain_mass(s):
    case = s["case"]
    n, n_q = case["ctx"], case["q_len"]
    q, k, v = s["q"], s["k"], s["v"]
    if s["k_new"] is not None:
        k[:, :, n:] = s["k_new"].transpose(1, 2)
        v[:, :, n:] = s["v_new"].transpose(1, 2)
    B, Hkv, N, d = k.shape
    G = q.shape[2] // Hkv
    rows = q.float().view(B, n_q, Hkv, G, d).permute(0, 2, 4, 1, 3).reshape(B, Hkv, d, n_q * G)
    z = torch.matmul(k.float(), rows) * (1.0 / math.sqrt(d))                        # [B, Hkv, N, rows]
    behind = torch.arange(N, device=k.device)[:, None] > n + torch.arange(n_q * G, device=k.device) // G
    z = z.masked_fill(behind, -math.inf)
    e = torch.exp(z - z.amax(2, keepdim=True))
    w = (e / e.sum(2, keepdim=True))
    out = torch.matmul(w.transpose(2, 3).contiguous(), v.float())                   # [B, Hkv, rows, d]
    out = out.view(B, Hkv, n_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, n_q, Hkv * G, d)
    mass = w.sum(3)
    mass[:, :, :n] += s["mass"]
    return dict(out=out.to(q.dtype), mass=mass, k_new=k[:, :, n:], v_new=v[:, :, n:])


def _plain_evict(s):
    case = s["case"]
    n, first, recent = case["rows"], case["first"], case["recent"]
    B, Hkv, _, d = s["k"].shape
    between = s["mass"][:, :, first:n - recent]
    order = torch.sort(between, dim=2, descending=True, stable=True).indices[:, :, :case["keep"] - first - recent]
    at = torch.arange(n, device="cuda").expand(B, Hkv, n)
    idx = torch.cat([at[:, :, :first], order.sort(dim=2).values + first, at[:, :, n - recent:]], 2)
    k, v = (torch.gather(s[x], 2, idx[..., None].expand(B, Hkv, case["keep"], d)) for x in ("k", "v"))
    return dict(idx=idx.to(torch.int32), k=k, v=v, mass=torch.gather(s["mass"], 2, idx))


def _plain_logprobs(s):
    case = s["case"]
    x = s["logits"].float()
    y = (x - x.amax(1, keepdim=True)) / case["temperature"]
    e = torch.exp(y)
    z = e.sum(1, keepdim=True)
    log_z = torch.log(z)
    tail = torch.where(e > 0, e * y, 0.0).sum(1, keepdim=True) / z
    got = dict(logprob=(torch.gather(y, 1, s["tokens"].long()[:, None]) - log_z)[:, 0], entropy=(log_z - tail)[:, 0])
    if case["top"]:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        got.update(top_ids=ids.to(torch.int32), top_logprobs=torch.gather(y, 1, ids) - log_z)
    return got


def run(s):
    if own:
        return _call(s)
    return {"mass": _plain_mass, "evict": _plain_evict, "logprobs": _plain_logprobs}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    es = ELEM_BYTES[case["dtype"]]
    if case["op"] == "logprobs":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * V * es + R * (12 + 8 * case["top"]), "flops": 5 * R * V}
    H, Hkv, d = HEADS[case["heads"]]
    B = case["batch"]
    if case["op"] == "evict":
        kept = B * Hkv * case["keep"]
        return {"bytes": B * Hkv * case["rows"] * 4 + kept * (2 * 2 * d * es + 8), "flops": B * Hkv * case["rows"]}
    n = case["ctx"] + case["q_len"]
    new = B * Hkv * case["q_len"] * 2 * d * es if case["append"] else 0
    return {"bytes": B * Hkv * n * (2 * d * es + 8) + 2 * B * H * case["q_len"] * d * es + new,
            "flops": B * H * case["q_len"] * n * (4 * d + 4)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "mass":
        n, (H, Hkv, d) = case["ctx"], HEADS[case["heads"]]
        G = H // Hkv
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        mass = torch.zeros(s["k"].shape[:3], dtype=torch.float64, device="cuda")
        mass[:, :, :n] = s["mass"].double()
        for b in range(case["batch"]):
            for hk in range(Hkv):
                k, v = s["k"][b, hk].double(), s["v"][b, hk].double()
                for i in range(case["q_len"]):
                    seen = n + i + 1
                    p = torch.softmax(s["q"][b, i, hk * G:(hk + 1) * G].double() @ k[:seen].T.contiguous() / math.sqrt(d), 1)
                    out[b, i, hk * G:(hk + 1) * G] = p @ v[:seen]
                    mass[b, hk, :seen] += p.sum(0)
        return dict(out=out, mass=mass, k_new=s["k"][:, :, n:].double(), v_new=s["v"][:, :, n:].double())
    if case["op"] == "evict":
        mass = s["mass"].double().cpu().numpy()
        B, Hkv, N = mass.shape
        first, last, k = case["first"], N - case["recent"], case["keep"] - case["first"] - case["recent"]
        idx = np.empty((B, Hkv, case["keep"]), np.int32)
        for b in range(B):
            for hk in range(Hkv):
                between = np.lexsort((np.arange(first, last), -mass[b, hk, first:last]))[:k] + first
                idx[b, hk] = np.concatenate([np.arange(first), np.sort(between), np.arange(last, N)])
        at = torch.from_numpy(idx).cuda()
        b, hk = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
        picked = {x: s[x][b, hk, at.long()] for x in ("k", "v", "mass")}
        if case["dtype"] != "fp8":
            picked.update({x: picked[x].double() for x in ("k", "v")})
        return dict(idx=at, **dict(picked, mass=picked["mass"].double()))
    R, n = case["rows"], case["top"]
    found = dict(logprob=torch.empty((R,), dtype=torch.float64), entropy=torch.empty((R,), dtype=torch.float64))
    if n:
        found.update(top_ids=torch.empty((R, n), dtype=torch.int32), top_logprobs=torch.empty((R, n), dtype=torch.float64))
    for r in range(R):
        x = s["logits"][r].double() / case["temperature"]
        p = torch.log_softmax(x, 0)
        found["logprob"][r] = p[int(s["tokens"][r])]
        alive = p[p > -math.inf]
        found["entropy"][r] = -(alive.exp() * alive).sum()
        if n:
            v = s["logits"][r].double()
            edge = torch.topk(v, n).values[-1]
            ids = torch.cat([torch.nonzero(v > edge)[:, 0], torch.nonzero(v == edge)[:n, 0]])
            ids = ids[torch.sort(v[ids], descending=True, stable=True).indices][:n]
            found["top_ids"][r], found["top_logprobs"][r] = ids.to(torch.int32), p[ids]
    return found
