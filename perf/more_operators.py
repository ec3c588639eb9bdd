"""From a prompt to a verified draft tree over a paged cache.

Verification and draft decoding start from a cache that something has filled.  Four operators fill it, keep its pages and verify
more than a chain over it:

  prefill   causal attention of whole prompts, packed one behind the other without padding, or of their next pieces over what the
            cache already holds, packed or in pages (hippo_prefill_attention, hippo_prefill_attention_paged)
  tree      attention of a tree of drafted tokens over a cache: a node sees the context, its ancestors and itself, and every
            sequence has a length of its own (hippo_tree_attention, hippo_tree_attention_paged)
  plan      the pages, block table rows, row slots and positions of a step's new tokens, and the pages that rejected or finished
            rows give back, from the requests' lengths (hippo_plan_pages)
  write     a step's K and V rows into the pages, by those slots (hippo_write_kv_paged)

Head layouts and cache lengths are those of synth_inputs.py's configurations (832, 16K, 33K and 4 x 37K rows); `draw` gives ragged
ones around them.

`own` False computes the operators in elementary torch operations, True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head dim) of the configurations
HEADS = {"4/2x64": (4, 2, 64), "14/2x64": (14, 2, 64), "28/4x128": (28, 4, 128), "64/8x128": (64, 8, 128)}
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
ELEM_BYTES = {"fp32": 4, "bf16": 2}


def _prefill(name, dtype, heads, new, ctx="0", page=0):
    """new, ctx: rows of each sequence that are attended from, and rows before them; page 0: packed K and V"""
    return dict(name=name, op="prefill", dtype=dtype, heads=heads, new=new, ctx=ctx, page=page)


def _tree(name, dtype, heads, nodes, ctx, page=0):
    return dict(name=name, op="tree", dtype=dtype, heads=heads, nodes=nodes, ctx=ctx, page=page)


def _plan(name, batch, longest, kind, page, spare):
    return dict(name=name, op="plan", batch=batch, longest=longest, kind=kind, page=page, spare=spare)


def _write(name, dtype, heads, tokens, source, page):
    return dict(name=name, op="write", dtype=dtype, heads=heads, tokens=tokens, source=source, page=page)


def listed():
    return [
        # the smallest prompt of the configurations, in fp32
        _prefill("prefill_fp32_832", "fp32", "4/2x64", "832"),
        # short questions that arrive together: latency, and sequences that end inside every tile
        _prefill("prefill_questions", "bf16", "28/4x128", "26,149,1,64,37,128,8,211,95,17,2,130"),
        # a draft model's prompts of very different lengths in one pass
        _prefill("prefill_ragged", "bf16", "14/2x64", "4224,832,1,1895,26,2600,513,149"),
        # a long video's prompt in one piece
        _prefill("prefill_16k", "bf16", "28/4x128", "16640"),
        # the next pieces of a batch of a large model's prompts, over what the pages already hold
        _prefill("prefill_pieces_37k", "bf16", "64/8x128", "512,300,768,511", "36608,20480,9216,30011", 16),
        # a small tree over a short fp32 cache: launches
        _tree("tree_fp32_832", "fp32", "4/2x64", 8, "832"),
        # a tree of the ordinary size over a video's whole cache
        _tree("tree_16k", "bf16", "28/4x128", 16, "16640"),
        # wide trees of a batch of a large model over pages, every request at its own length: the most bytes
        _tree("tree_paged_37k", "bf16", "64/8x128", 64, "37120,16640,33280,29001", 16),
        # a decoding step of many requests: a few tokens each, rejected rows given back
        _plan("plan_step", 256, 16640, "step", 16, 1.0),
        # prompts admitted together
        _plan("plan_prompts", 48, 8192, "prompts", 16, 0.7),
        # the accepted path of each of 64 trees: few rows, picked from the trees' rows
        _write("write_paths", "bf16", "28/4x128", 256, "picked", 16),
        # a prompt's rows, out of a fused projection's output
        _write("write_16k", "bf16", "28/4x128", 16640, "fused", 16),
    ]


# ---------------------------------------------------------------------------------------------------------------
# drawn cases
# ---------------------------------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(numbers):
    return ",".join(str(n) for n in numbers)


def _draw_once(rng):
    op = rng.choice(["prefill", "prefill", "tree", "tree", "plan", "write"])
    dtype, heads = rng.choice(["bf16", "bf16", "bf16", "fp32"]), rng.choice(sorted(HEADS))
    page = rng.choice([16, 16, 32, 64, 256])
    if op == "prefill":
        n = rng.choice([1, 1, 2, 3, 5, rng.randint(6, 40)])
        new = [_log_int(rng, 1, 16640) for _ in range(n)]
        kind = rng.choice(["own", "own", "behind", "paged"])
        ctx = [0] if kind == "own" else [_log_int(rng, 1, 37120) - 1 for _ in range(n)]
        return dict(op=op, dtype=dtype, heads=heads, new=_text(new), ctx=_text(ctx), page=page if kind == "paged" else 0)
    if op == "tree":
        ctx = [_log_int(rng, 16, 37120) for _ in range(rng.choice([1, 1, 2, 3, 4]))]
        return dict(op=op, dtype=dtype, heads=heads, nodes=rng.choice([2, 8, 16, 32, 64, rng.randint(1, 64)]), ctx=_text(ctx),
                    page=rng.choice([0, page]))
    if op == "plan":
        return dict(op=op, batch=_log_int(rng, 1, 512), longest=_log_int(rng, 64, 16640), kind=rng.choice(["step", "step", "prompts"]),
                    page=page, spare=rng.choice([1.0, 1.0, 0.6]))
    return dict(op=op, dtype=dtype, heads=heads, tokens=_log_int(rng, 1, 33000), source=rng.choice(["fused", "plain", "picked"]), page=page)


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (1e14 if case.get("dtype") == "fp32" else 1e15)


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("prefill", "tree", "plan", "write")}
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most[case["op"]]:
            return case


def _numbers(text):
    return [int(x) for x in text.split(",")]


def _lengths(case):
    """(new rows, rows before them) of each sequence"""
    new, ctx = _numbers(case["new"]), _numbers(case["ctx"])
    return new, ctx if len(ctx) == len(new) else ctx * len(new)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _offsets(lens):
    return _int32([0] + list(np.cumsum(lens)))


def _pool(g, lens, page, Hkv, d, dtype):
    """Pools whose pages are dealt to the sequences in random order, and the block table: [pages, page, Hkv, d] twice, [B, most]"""
    need = [-(-n // page) for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(lens), max(need) + 1), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return _rows(g, total, page, Hkv, d, dtype=dtype), _rows(g, total, page, Hkv, d, dtype=dtype), table


def _rows(g, first, *rest, dtype, factor=1.0):
    """normal entries, made in pieces"""
    x = torch.empty((first,) + rest, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, math.prod(rest)))
    for i in range(0, first, step):
        x[i:i + step] = _normal(g, min(step, first - i), *rest) * factor
    return x


def _prepare_prefill(case, g):
    H, Hkv, d = HEADS[case["heads"]]
    t = TORCH_DTYPE[case["dtype"]]
    new, ctx = _lengths(case)
    both = [a + b for a, b in zip(new, ctx)]
    s = dict(new=new, ctx=ctx, q=_rows(g, sum(new), H, d, dtype=t, factor=1.3), cu_q=_offsets(new), table=None, cu_k=None)
    if case["page"]:
        s["k"], s["v"], s["table"] = _pool(g, both, case["page"], Hkv, d, t)
        s["kv_lens"] = _int32(both)
    else:
        s["k"], s["v"] = (_rows(g, sum(both), Hkv, d, dtype=t) for _ in range(2))
        if any(ctx):
            s["cu_k"] = _offsets(both)
    return s


def _prepare_tree(case, g):
    """A tree grows where the draft model is unsure: a node's parent is near behind it.  Elements of a batch whose tree is smaller
    are padded with nodes that are none (-2)."""
    H, Hkv, d = HEADS[case["heads"]]
    t, n, ctx = TORCH_DTYPE[case["dtype"]], case["nodes"], _numbers(case["ctx"])
    B = len(ctx)
    s = dict(ctx=ctx, q=_rows(g, B, n, H, d, dtype=t, factor=1.3), ctx_lens=_int32(ctx), table=None)
    if case["page"]:
        s["k"], s["v"], s["table"] = _pool(g, [c + n for c in ctx], case["page"], Hkv, d, t)
    else:
        s["k"], s["v"] = (_rows(g, B, Hkv, max(ctx) + n, d, dtype=t) for _ in range(2))
    node = torch.arange(n, device="cuda")
    back = (torch.rand((B, n), generator=g, device="cuda") ** 2 * (node + 1).clamp(max=12)).long()
    parents = (node - 1 - back).clamp(min=-1)
    size = n - torch.randint(0, n // 4 + 1, (B, 1), generator=g, device="cuda") * (torch.arange(B, device="cuda")[:, None] > 0)
    s["parents"] = torch.where(node < size, parents, -2).to(torch.int32)
    return s


def _prepare_plan(case, g):
    """Requests in the middle of their answers (step: some take a few tokens more, some give back what was rejected, some are
    done) or with a prompt to admit; `spare`: how much of the pages that they ask for is free."""
    B, page, longest = case["batch"], case["page"], case["longest"]
    u = lambda *shape: torch.rand(shape, generator=g, device="cuda")            # noqa: E731
    if case["kind"] == "step":
        ctx = torch.exp(u(B) * math.log(longest)).long()
        new = torch.randint(1, 9, (B,), generator=g, device="cuda")
        new = torch.where(u(B) < 0.3, -torch.randint(0, 64, (B,), generator=g, device="cuda"), new)
        new = torch.where(u(B) < 0.05, -ctx, new)
    else:
        ctx = torch.where(u(B) < 0.25, torch.randint(0, longest + 1, (B,), generator=g, device="cuda"), 0)
        new = torch.exp(u(B) * math.log(longest)).long()
    held, want = -(-ctx // page), -(-(ctx + new).clamp(min=0) // page)
    columns = (1 if case["kind"] == "step" else 2) * -(-longest // page) + 2
    n_pool = B * columns
    order = torch.randperm(n_pool, generator=g, device="cuda").to(torch.int32)
    column = torch.arange(columns, device="cuda")
    taken = column < held[:, None]
    at = (held.cumsum(0) - held)[:, None] + column
    table = torch.where(taken, order[torch.where(taken, at, 0)], -1)
    n_free = int(case["spare"] * int((want - held).clamp(min=0).sum())) + (64 if case["spare"] >= 1 else 0)
    n_free = min(n_free, n_pool - int(held.sum()))
    free = torch.full((n_pool,), -1, dtype=torch.int32, device="cuda")
    free[:n_free] = order[int(held.sum()):int(held.sum()) + n_free]
    # slots for the most tokens that such a step brings
    most = 8 * B if case["kind"] == "step" else B * longest // 4 + 1
    return dict(ctx=ctx.to(torch.int32), new=new.to(torch.int32), table=table.contiguous(), free=free, n_free=_int32([n_free]),
                most=most)


def _prepare_write(case, g):
    H, Hkv, d = HEADS[case["heads"]]
    t, n, page = TORCH_DTYPE[case["dtype"]], case["tokens"], case["page"]
    pages = -(-n // page) + 5
    s = dict(k_pool=_rows(g, pages, page, Hkv, d, dtype=t), v_pool=_rows(g, pages, page, Hkv, d, dtype=t), rows=None)
    if case["source"] == "fused":       # K and V heads behind the query heads of one projection's output
        fused = _rows(g, n, H + 2 * Hkv, d, dtype=t)
        s["k"], s["v"] = fused[:, H:H + Hkv], fused[:, H + Hkv:]
    else:
        made = n if case["source"] == "plain" else 4 * n
        s["k"], s["v"] = (_rows(g, made, Hkv, d, dtype=t) for _ in range(2))
        if case["source"] == "picked":
            s["rows"] = (4 * torch.arange(n, device="cuda") + torch.randint(0, 4, (n,), generator=g, device="cuda")).to(torch.int32)
    # consecutive rows of pages in random order; the last few tokens of a padded step have no slot
    order = torch.randperm(pages, generator=g, device="cuda")
    token = torch.arange(n, device="cuda") + 5
    slots = order[token // page] * page + token % page
    s["slots"] = torch.where(token - 5 < n - n // 50, slots, -1).to(torch.int32)
    return s


_PREPARE = {"prefill": _prepare_prefill, "tree": _prepare_tree, "plan": _prepare_plan, "write": _prepare_write}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return dict(case=case, **_PREPARE[case["op"]](case, g))


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _call(s):
    """The pass as the library's user writes it."""
    import paper_2601_08273_amd as h
    case = s["case"]
    if case["op"] == "prefill":
        if s["table"] is not None:
            return h.hippo_prefill_attention_paged(s["q"], s["k"], s["v"], s["table"], s["cu_q"], s["kv_lens"])
        return h.hippo_prefill_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"])
    if case["op"] == "tree":
        if s["table"] is not None:
            return h.hippo_tree_attention_paged(s["q"], s["k"], s["v"], s["table"], s["parents"], s["ctx_lens"])
        return h.hippo_tree_attention(s["q"], s["k"], s["v"], s["parents"], s["ctx_lens"])
    if case["op"] == "plan":
        slots, positions, cu_q, kv_lens, n_free = h.hippo_plan_pages(s["ctx"], s["new"], s["table"], s["free"], s["n_free"],
                                                                     case["page"], s["most"])
        return dict(slots=slots, positions=positions, cu_q=cu_q, kv_lens=kv_lens, n_free=n_free, table=s["table"], free=s["free"])
    h.hippo_write_kv_paged(s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"], rows=s["rows"])
    return dict(k=s["k_pool"], v=s["v_pool"])


def _weighted(q, k, v, hidden):
    """q [.., Hkv, rows, d], k and v [.., Hkv, n, d], hidden [.., 1, rows, n]: softmax over what is not hidden, times v; rows
    that see nothing give zeros.  In place where it can be: the logits of a long prompt are most of the memory."""
    z = torch.matmul(q.float(), (k.float() * (1.0 / math.sqrt(q.shape[-1]))).transpose(-1, -2).contiguous())
    z.masked_fill_(hidden, -math.inf)
    z.sub_(z.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = z.sum(-1, keepdim=True)
    return torch.matmul(z, v.float().contiguous()) / torch.where(total > 0, total, 1.0)


def _plain_prompt(q, k, v):
    """one sequence: q [n, H, d], k and v [m, Hkv, d], the last rows of both the same"""
    n, H, d = q.shape
    m, Hkv, _ = k.shape
    G = H // Hkv
    rows = q.view(n, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, n * G, d)
    sees = m - n + torch.arange(n * G, device=q.device)[:, None] // G
    out = _weighted(rows, k.transpose(0, 1), v.transpose(0, 1), torch.arange(m, device=q.device) > sees)
    return out.view(Hkv, n, G, d).permute(1, 0, 2, 3).reshape(n, H, d).to(q.dtype)


def _in_order(pool, pages):
    """pages [.., columns] of a pool [pages, page, Hkv, d], one behind the other: [.., columns * page, Hkv, d]"""
    return pool[pages.long()].flatten(-4, -3)


def _plain_prefill(s):
    new, both = s["new"], [a + b for a, b in zip(s["new"], s["ctx"])]
    if s["table"] is None:
        ks, vs = torch.split(s["k"], both), torch.split(s["v"], both)
    else:
        ks, vs = ([_in_order(s[x], table)[:n] for table, n in zip(s["table"], both)] for x in ("k", "v"))
    return torch.cat([_plain_prompt(*x) for x in zip(torch.split(s["q"], new), ks, vs)])


def _plain_tree(s):
    q, ctx, parents = s["q"], s["ctx_lens"].long()[:, None, None], s["parents"].long()
    B, n, H, d = q.shape
    node = torch.arange(n, device=q.device)
    # a node reaches its ancestors and itself: (I + parent)^n; what is padding reaches nothing and is reached by nothing
    step = (parents[:, :, None] == node).float() + torch.eye(n, device=q.device)
    there = parents >= -1
    reach = (torch.linalg.matrix_power(step, n) > 0) & there[:, :, None] & there[:, None, :]
    if s["table"] is None:
        k, v = s["k"], s["v"]
    else:
        k, v = (_in_order(s[x], s["table"]).transpose(1, 2) for x in ("k", "v"))
    Hkv, N = k.shape[1:3]
    G = H // Hkv
    behind = torch.arange(N, device=q.device) - ctx                                # [B, 1, N]
    inside = torch.gather(reach, 2, behind.clamp(0, n - 1).expand(B, n, N)) & (behind >= 0) & (behind < n)
    sees = ((behind < 0) & there[:, :, None]) | inside                              # [B, n, N]
    hidden = ~sees.repeat_interleave(G, 1)[:, None]
    rows = q.view(B, n, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, d)
    out = _weighted(rows, k, v, hidden)
    return out.view(B, Hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, H, d).to(q.dtype)


def _plain_plan(s):
    page, most = s["case"]["page"], s["most"]
    ctx, new, n_free = s["ctx"].long(), s["new"].long(), s["n_free"].long()
    B, columns = s["table"].shape
    n_pool = s["free"].numel()
    held, after = -(-ctx // page), (ctx + new).clamp(min=0)
    want = -(-after // page)
    column = torch.arange(columns, device="cuda")
    # what is given back goes on the stack of free pages, in the order of the table
    given = ((column >= want[:, None]) & (column < held[:, None])).flatten()
    at = torch.where(given, n_free + given.cumsum(0) - 1, n_pool)
    free = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter(0, at, s["table"].flatten())[:n_pool]
    available = n_free + given.sum()
    # requests are admitted while pages and token slots last
    grows = (new >= 0) & (want <= columns)
    pages, tokens = torch.where(grows, (want - held).clamp(min=0), 0), torch.where(grows, new, 0)
    admitted = grows & ((pages == 0) | (pages.cumsum(0) <= available)) & ((tokens == 0) | (tokens.cumsum(0) <= most))
    pages, tokens = pages * admitted, tokens * admitted
    taken = (column >= held[:, None]) & (column < want[:, None]) & admitted[:, None]
    number = (pages.cumsum(0) - pages)[:, None] + column - held[:, None]
    table = torch.where(taken, free[(available - 1 - torch.where(taken, number, 0)).clamp(0, n_pool - 1)], s["table"])
    kv_lens = torch.where(admitted | (new < 0), after, ctx)
    ends = tokens.cumsum(0)
    token = torch.arange(most, device="cuda")
    b = torch.searchsorted(ends, token, right=True).clamp(max=B - 1)
    position = ctx[b] + token - (ends - tokens)[b]
    slot = table[b, (position // page).clamp(0, columns - 1)] * page + position % page
    real = token < ends[-1]
    cu_q = torch.cat([ends.new_zeros(1), ends])
    found = dict(slots=torch.where(real, slot, -1), positions=torch.where(real, position, -1), cu_q=cu_q, kv_lens=kv_lens,
                 n_free=available - pages.sum(), table=table, free=free)
    return {name: x.to(torch.int32) for name, x in found.items()}


def _plain_write(s):
    real = s["slots"] >= 0
    slots = s["slots"][real].long()
    rows = torch.arange(len(s["slots"]), device="cuda") if s["rows"] is None else s["rows"].long()
    s["k_pool"].flatten(0, 1)[slots] = s["k"][rows[real]]
    s["v_pool"].flatten(0, 1)[slots] = s["v"][rows[real]]
    return dict(k=s["k_pool"], v=s["v_pool"])


def run(s):
    if own:
        return _call(s)
    return {"prefill": _plain_prefill, "tree": _plain_tree, "plan": _plain_plan, "write": _plain_write}[s["case"]["op"]](s)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "plan":
        # lengths, a token's slot and position, a page's number read and written
        tokens = case["batch"] * (case["longest"] // 4 if case["kind"] == "prompts" else 8) + 1
        return {"bytes": int(case["batch"] * 16 + tokens * (8 + 8 / case["page"])), "flops": int(10 * (case["batch"] + tokens))}
    es = ELEM_BYTES[case["dtype"]]
    H, Hkv, d = HEADS[case["heads"]]
    if case["op"] == "write":
        return {"bytes": case["tokens"] * (4 * Hkv * d * es + 4), "flops": 0}
    if case["op"] == "prefill":
        new, ctx = _lengths(case)
        rows, keys = sum(new), sum(new) + sum(ctx)
        pairs = sum(n * c + n * (n + 1) // 2 for n, c in zip(new, ctx))
    else:
        ctx, n = _numbers(case["ctx"]), case["nodes"]
        rows, keys = len(ctx) * n, sum(ctx) + len(ctx) * n
        pairs = sum(n * c + n * min(n, 6) for c in ctx)
    return {"bytes": 2 * rows * H * d * es + 2 * keys * Hkv * d * es, "flops": pairs * H * (4 * d + 4)}


def _exact_rows(q, k, v, sees):
    """q [r, G, d], k and v [n, d], sees [r, n] truth values: in 64 bits, a few hundred rows at a time"""
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    kt, v = (k.double() / math.sqrt(q.shape[2])).T.contiguous(), v.double()
    for i in range(0, q.shape[0], 512):
        z = (q[i:i + 512].double() @ kt).masked_fill(~sees[i:i + 512, None], -math.inf)
        out[i:i + 512] = torch.nan_to_num(torch.softmax(z, 2), nan=0.0) @ v
    return out


def _exact_prefill(s):
    new, ctx = s["new"], s["ctx"]
    H, Hkv, d = HEADS[s["case"]["heads"]]
    G, page = H // Hkv, s["case"]["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    at_q = at_k = 0
    for b, (n, c) in enumerate(zip(new, ctx)):
        if page:
            row = torch.arange(n + c, device="cuda")
            place = (s["table"][b, row // page].long(), row % page)
        else:
            place = (torch.arange(at_k, at_k + n + c, device="cuda"),)
        sees = torch.ones((n, n + c), dtype=torch.bool, device="cuda").tril(c)
        for hk in range(Hkv):
            heads = slice(hk * G, (hk + 1) * G)
            out[at_q:at_q + n, heads] = _exact_rows(s["q"][at_q:at_q + n, heads], s["k"][place][:, hk], s["v"][place][:, hk], sees)
        at_q, at_k = at_q + n, at_k + n + c
    return out


def _exact_tree(s):
    H, Hkv, d = HEADS[s["case"]["heads"]]
    G, page = H // Hkv, s["case"]["page"]
    B, n = s["parents"].shape
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    parents = s["parents"].tolist()
    for b, c in enumerate(s["ctx"]):
        sees = np.zeros((n, c + n), bool)
        for i in range(n):
            if parents[b][i] >= -1:
                sees[i, :c] = True
            j = i
            while parents[b][i] >= -1 and j >= 0:
                sees[i, c + j] = True
                j = parents[b][j]
        sees = torch.from_numpy(sees).cuda()
        row = torch.arange(c + n, device="cuda")
        for hk in range(Hkv):
            if page:
                k, v = (s[x][s["table"][b, row // page].long(), row % page, hk] for x in ("k", "v"))
            else:
                k, v = (s[x][b, hk, :c + n] for x in ("k", "v"))
            heads = slice(hk * G, (hk + 1) * G)
            out[b, :, heads] = _exact_rows(s["q"][b, :, heads], k, v, sees)
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    if case["op"] == "prefill":
        return _exact_prefill(s)
    if case["op"] == "tree":
        return _exact_tree(s)
    slots = s["slots"].cpu().numpy()
    at = np.nonzero(slots >= 0)[0]
    source = at if s["rows"] is None else s["rows"].cpu().numpy()[at]
    found = {}
    for name in ("k", "v"):
        pool, new = s[name + "_pool"].double().cpu().numpy(), s[name].double().cpu().numpy()
        page = pool.shape[1]
        pool[slots[at] // page, slots[at] % page] = new[source]
        found[name] = torch.from_numpy(pool)
    return found
