"""GPU: hippo_plan_pages against a plain loop over the requests, hippo_write_kv_paged against indexing, and a run of a prompt and a
draft tree over the pages that they make."""
import numpy as np
import pytest
import torch

from attention_reference import check
from test_gpu_prefill import TYPES, reference as prefill_reference, rows
from test_gpu_tree import int32, reference as tree_reference, some_tree

pytestmark = pytest.mark.gpu


def plan(ctx, new, table, free, n_free, page, most):
    """the definition, request by request"""
    table, free, (B, columns) = table.copy(), free.copy(), table.shape
    pages = lambda n: -(-n // page)                                          # noqa: E731
    top = n_free = min(max(n_free, 0), len(free))
    ctx = [max(c, 0) for c in ctx]
    after = [max(c + n, 0) for c, n in zip(ctx, new)]
    for b in range(B):
        if new[b] < 0:
            for i in range(min(pages(after[b]), columns), min(pages(ctx[b]), columns)):
                if top < len(free):
                    free[top] = table[b, i]
                    top += 1
    available, asked_pages, asked_tokens = top, 0, 0
    kv, cu, slots, positions = list(ctx), [0], [], []
    for b in range(B):
        if new[b] < 0:
            kv[b] = after[b]
        elif pages(after[b]) <= columns:
            need = max(pages(after[b]) - pages(ctx[b]), 0)
            asked_pages, asked_tokens = asked_pages + need, asked_tokens + new[b]
            if (need == 0 or asked_pages <= available) and (new[b] == 0 or asked_tokens <= most):
                for i in range(pages(ctx[b]), pages(after[b])):
                    top -= 1
                    table[b, i] = free[top]
                kv[b] = after[b]
                for r in range(ctx[b], after[b]):
                    pg = table[b, r // page]
                    slots.append(pg * page + r % page if 0 <= pg < len(free) else -1)
                    positions.append(r)
        cu.append(len(slots))
    pad = [-1] * (most - len(slots))
    return dict(slots=slots + pad, positions=positions + pad, cu_q=cu, kv_lens=kv, n_free=[top], table=table, free=free)


def run(h, ctx, new, table, free, n_free, page, most):
    t, f = int32(table), int32(free)
    got = h.hippo_plan_pages(int32(ctx), int32(new), t, f, int32([n_free]), page, most)
    return dict(zip(("slots", "positions", "cu_q", "kv_lens", "n_free"), got), table=t, free=f)


def compare(got, want, what=""):
    for name, x in want.items():
        np.testing.assert_array_equal(got[name].cpu().numpy(), np.asarray(x, dtype=np.int64).reshape(got[name].shape), err_msg="%s %s" % (what, name))


def state(rng, B, longest, page, kind, spare):
    if kind == "step":
        ctx = rng.integers(0, longest + 1, B)
        new = np.where(rng.random(B) < 0.4, -rng.integers(0, 3 * page, B), rng.integers(0, 9, B))
        new = np.where(rng.random(B) < 0.1, -ctx - rng.integers(0, 2, B), new)
    else:
        ctx = np.where(rng.random(B) < 0.3, rng.integers(0, longest + 1, B), 0)
        new = rng.integers(0, longest + 1, B)
    columns = -(-longest // page) + (1 if kind == "step" else int(rng.integers(0, 4)))
    held = -(-ctx // page)
    n_pool = int(held.sum()) + int(spare * max(1, (-(-np.maximum(ctx + new, 0) // page) - held).clip(0).sum())) + 1
    order = rng.permutation(n_pool)
    table = np.full((B, columns), -1, np.int64)
    at = 0
    for b in range(B):
        n = min(held[b], columns)
        table[b, :n] = order[at:at + n]
        at += held[b]
    free = np.full(n_pool, -1, np.int64)
    n_free = n_pool - int(held.sum())
    free[:n_free] = order[int(held.sum()):]
    return [int(x) for x in ctx], [int(x) for x in new], table, free, n_free


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 300, 1024, 1025])
@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("kind,spare", [("step", 1.0), ("step", 0.3), ("prompts", 1.0), ("prompts", 0.5), ("prompts", 0.0)])
def test_plans(hippo, B, page, kind, spare):
    for seed in range(3):
        rng = np.random.default_rng([seed, B, page])
        s = state(rng, B, 600, page, kind, spare)
        total = sum(n for n in s[1] if n > 0)
        for most in {0, max(1, total), max(1, total // 2), total + 37}:
            compare(run(hippo, *s, page, most), plan(*s, page, most), "%s %s %s" % (seed, B, most))


def test_a_large_plan(hippo):
    rng = np.random.default_rng(4)
    s = state(rng, 4096, 700, 16, "prompts", 0.8)
    most = sum(s[1])
    compare(run(hippo, *s, 16, most), plan(*s, 16, most))


@pytest.mark.parametrize("ctx,new,n_free", [([0], [0], 5), ([5], [-5], 0), ([5], [-9], 0), ([-3, 7], [4, 9], 5), ([0, 0], [2 ** 31 - 1, 3], 5),
                                            ([2 ** 31 - 1, 3], [1, 2], 5), ([2 ** 31 - 1, 3], [-(2 ** 31), 2], 5), ([64, 0], [0, 64], 4),
                                            ([64, 0], [-64, 64], 0), ([63], [1], 0), ([64], [1], 0), ([17, 5], [3, 3], -4), ([0], [3], 100)])
def test_edges(hippo, ctx, new, n_free):
    table = np.arange(len(ctx) * 4).reshape(len(ctx), 4) % 5
    free = np.array([4, 3, 2, 1, 0, 9, 9, 9])
    compare(run(hippo, ctx, new, table, free, n_free, 16, 80), plan(ctx, new, table, free, n_free, 16, 80))


def test_pages_that_are_none_get_no_slot(hippo):
    got = run(hippo, [3], [40], np.array([[-7, 0, 0, 0]]), np.array([2 ** 31 - 1, 1, 2 ** 30]), 3, 16, 50)
    compare(got, plan([3], [40], np.array([[-7, 0, 0, 0]]), np.array([2 ** 31 - 1, 1, 2 ** 30]), 3, 16, 50))


def test_a_step_may_be_repeated(hippo):
    rng = np.random.default_rng(6)
    ctx, new, table, free, n_free = state(rng, 50, 300, 16, "step", 1.0)
    t, f, c, n, k = int32(table), int32(free), int32(ctx), int32(new), int32([n_free])
    first = [x.clone() for x in hippo.hippo_plan_pages(c, n, t, f, k, 16, 400)] + [t.clone(), f.clone()]
    again = list(hippo.hippo_plan_pages(c, n, t, f, k, 16, 400)) + [t, f]
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_inputs_beside_outputs(hippo):
    """all of a plan in one buffer, an input next to an output everywhere"""
    B, columns, n_pool, most, page = 3, 4, 9, 40, 16
    ctx, new, n_free = [20, 5, 40], [15, 30, -10], 4
    table = [[8, 7, -1, -1], [6, -1, -1, -1], [5, 4, 3, -1]]
    free = [0, 1, 2, 5, -1, -1, -1, -1, -1]
    sizes = [("table", B * columns), ("ctx", B), ("slots", most), ("new", B), ("free", n_pool), ("n_free", 1), ("cu_q", B + 1), ("positions", most),
             ("kv_lens", B), ("left", 1)]
    whole, at, part = torch.full((sum(n for _, n in sizes),), -7, dtype=torch.int32, device="cuda"), 0, {}
    for name, n in sizes:
        part[name], at = whole[at:at + n], at + n
    for name, x in (("table", sum(table, [])), ("ctx", ctx), ("new", new), ("free", free), ("n_free", [n_free])):
        part[name].copy_(int32(x))
    part["table"] = part["table"].view(B, columns)
    hippo.hippo_plan_pages(part["ctx"], part["new"], part["table"], part["free"], part["n_free"], page, most, slots_out=part["slots"],
                           positions_out=part["positions"], cu_q_out=part["cu_q"], kv_lens_out=part["kv_lens"], n_free_out=part["left"])
    want = plan(ctx, new, np.array(table), np.array(free), n_free, page, most)
    compare(dict(part, n_free=part["left"]), want)
    assert part["ctx"].tolist() == ctx and part["new"].tolist() == new and part["n_free"].tolist() == [n_free]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hkv,d,page", [(1, 64, 16), (2, 64, 32), (4, 128, 16), (8, 128, 256), (3, 64, 64)])
@pytest.mark.parametrize("T", [0, 1, 3, 4, 5, 333])
def test_writes(hippo, dtype, Hkv, d, page, T):
    g = torch.Generator(device="cuda").manual_seed(T + Hkv)
    pages = -(-T // page) + 2
    pools = [rows(g, pages, page, Hkv, d, dtype=dtype) for _ in range(2)]
    fused = rows(g, T, 3 + 2 * Hkv, d, dtype=dtype)
    news = [fused[:, 3:3 + Hkv], fused[:, 3 + Hkv:]]
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T].to(torch.int32)
    if T > 3:
        slots[1], slots[2] = -1, pages * page                              # no such slots
        slots[3] = 2 ** 31 - 1
    want = [p.clone() for p in pools]
    ok = (slots >= 0) & (slots < pages * page)
    for p, x in zip(want, news):
        p.view(-1, Hkv, d)[slots[ok].long()] = x[ok]
    assert hippo.hippo_write_kv_paged(*news, slots, *pools) is None
    assert all(torch.equal(a, b) for a, b in zip(pools, want))
    pick = torch.randint(0, max(T, 1), (T,), generator=g, device="cuda").to(torch.int32)
    if T > 4:
        pick[0], pick[4] = -1, T
    ok &= (pick >= 0) & (pick < T)
    for p, x in zip(want, news):
        p.view(-1, Hkv, d)[slots[ok].long()] = x[pick[ok].long()]
    hippo.hippo_write_kv_paged(*news, slots, *pools, rows=pick)
    assert all(torch.equal(a, b) for a, b in zip(pools, want))


def test_pools_of_other_strides(hippo):
    """heads before rows inside a page, pages apart; what lies between is left alone"""
    g = torch.Generator(device="cuda").manual_seed(1)
    base = [torch.full((5, 2, 4, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pools = [x[:, 1].transpose(1, 2) for x in base]                        # [5, 16, 4, 64]
    news = [rows(g, 20, 4, 64, dtype="bf16") for _ in range(2)]
    slots = torch.randperm(80, generator=g, device="cuda")[:20].to(torch.int32)
    hippo.hippo_write_kv_paged(*news, slots, *pools)
    for x, pool, new in zip(base, pools, news):
        assert (x[:, 0] == 7).all()
        assert torch.equal(pool[(slots // 16).long(), (slots % 16).long()], new)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_pool_of_one_page(hippo, dtype):
    """heads first inside the page: the stride from page to page that a view of it has is shorter than a page"""
    g = torch.Generator(device="cuda").manual_seed(23)
    page, H, Hkv, d, n = 64, 8, 4, 64, 50
    k_pool, v_pool = (torch.zeros((Hkv, page, d), dtype=TYPES[dtype], device="cuda").transpose(0, 1)[None] for _ in range(2))
    k, v, q = rows(g, n, Hkv, d, dtype=dtype), rows(g, n, Hkv, d, dtype=dtype), rows(g, n, H, d, dtype=dtype)
    hippo.hippo_write_kv_paged(k, v, torch.arange(n, dtype=torch.int32, device="cuda"), k_pool, v_pool)
    assert torch.equal(k_pool[0, :n], k) and torch.equal(v_pool[0, :n], v) and not k_pool[0, n:].any()
    table, cu = int32([[0]]), int32([0, n])
    out = hippo.hippo_prefill_attention_paged(q, k_pool, v_pool, table, cu, int32([n]))
    assert torch.equal(out, hippo.hippo_prefill_attention_paged(q, k_pool.contiguous(), v_pool.contiguous(), table, cu, int32([n])))
    ref = prefill_reference(q, k, v, [n], [n])
    check(out, ref[0], ref[1])
    parents = int32([some_tree(10, 1)])
    out = hippo.hippo_tree_attention_paged(q[None, :10], k_pool, v_pool, table, parents, n - 10)
    assert torch.equal(out, hippo.hippo_tree_attention_paged(q[None, :10], k_pool.contiguous(), v_pool.contiguous(), table, parents, n - 10))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_token_with_k_and_v_of_other_tensors(hippo, dtype):
    """K as a kernel of its own wrote it, V a slice of the projection; then one KV head, whose tokens are as far apart in both"""
    g = torch.Generator(device="cuda").manual_seed(24)
    page, H, Hkv, d = 16, 8, 2, 64
    k_pool, v_pool = (torch.zeros((3, page, Hkv, d), dtype=TYPES[dtype], device="cuda") for _ in range(2))
    k, v = rows(g, 1, Hkv, d, dtype=dtype), rows(g, 1, H + 2 * Hkv, d, dtype=dtype)[:, H + Hkv:]
    q = rows(g, 1, H, d, dtype=dtype)
    hippo.hippo_write_kv_paged(k, v, int32([21]), k_pool, v_pool)
    assert torch.equal(k_pool[1, 5], k[0]) and torch.equal(v_pool[1, 5], v[0])
    assert not k_pool.flatten(0, 1)[torch.arange(48) != 21].any() and not v_pool.flatten(0, 1)[torch.arange(48) != 21].any()
    out = hippo.hippo_prefill_attention(q, k, v, int32([0, 1]))
    ref = prefill_reference(q, k, v, [1], [1])
    check(out, ref[0], ref[1])
    k, v, q = rows(g, 30, 1, d, dtype=dtype), rows(g, 1, 30, d, dtype=dtype).transpose(0, 1), rows(g, 30, H, d, dtype=dtype)
    out = hippo.hippo_prefill_attention(q, k, v, int32([0, 30]))
    ref = prefill_reference(q, k, v, [30], [30])
    check(out, ref[0], ref[1])


def test_a_pool_beyond_32_bit_offsets(hippo):
    pool = [torch.zeros((70000 * 16, 16, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]     # 4.6 GB each
    g = torch.Generator(device="cuda").manual_seed(2)
    news = [rows(g, 3, 2, 64, dtype="bf16") for _ in range(2)]
    slots = torch.tensor([70000 * 256 - 1, 5, 70000 * 200], dtype=torch.int32, device="cuda")
    hippo.hippo_write_kv_paged(*news, slots, *pool)
    for p, x in zip(pool, news):
        assert torch.equal(p.view(-1, 2, 64)[slots.long()], x)


@pytest.mark.parametrize("dtype,heads,page", [("bf16", (28, 4, 128), 16), ("fp32", (4, 2, 64), 32)])
@pytest.mark.parametrize("captured", [False, True])
def test_prompts_and_trees_over_the_pages_that_they_make(hippo, dtype, heads, page, captured):
    """Prompts in two pieces, a tree for each, the accepted paths kept, a second tree: every step is a plan, a write, an attention.
    The rows of each request are kept on the side, and every attention is checked against them."""
    h, (H, Hkv, d) = hippo, heads
    g = torch.Generator(device="cuda").manual_seed(3)
    B, columns, n_pool = 3, 20, 40
    table = torch.zeros((B, columns), dtype=torch.int32, device="cuda")
    free, n_free = torch.randperm(n_pool, generator=g, device="cuda").to(torch.int32), int32([n_pool])
    lens = int32([0] * B)
    k_pool, v_pool = (torch.full((n_pool, page, Hkv, d), float("nan"), dtype=TYPES[dtype], device="cuda") for _ in range(2))
    held = [[[], []] for _ in range(B)]                                    # K and V rows of each request

    def cache(x, b):
        return torch.stack(held[b][x]) if held[b][x] else torch.zeros((0, Hkv, d), dtype=TYPES[dtype], device="cuda")

    def step(new, most, attention):
        """plan and write, then attention(plan): as one graph where captured"""
        nonlocal n_free, lens
        T = sum(max(n, 0) for n in new)
        k, v = (rows(g, most, Hkv, d, dtype=dtype) for _ in range(2))
        add = int32(new)

        def calls():
            p = h.hippo_plan_pages(lens, add, table, free, n_free, page, most)
            h.hippo_write_kv_paged(k, v, p[0], k_pool, v_pool)
            return p, attention(p)
        if captured:
            before = [x.clone() for x in (table, free)]
            calls()                                                        # (the stack may be popped again: n_free is the old one)
            for x, y in zip((table, free), before):
                x.copy_(y)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                p, out = calls()
            for _ in range(2):
                graph.replay()
        else:
            p, out = calls()
        at = 0
        for b, n in enumerate(new):
            for x, rows_ in zip((0, 1), (k, v)):
                if n < 0:
                    held[b][x] = held[b][x][:n]
                else:
                    held[b][x] += list(rows_[at:at + n])
            at += max(n, 0)
        assert at == T and p[3].tolist() == [len(x[0]) for x in held]
        lens, n_free = p[3].clone(), p[4].clone()
        return out, (k, v)

    for new in ([37, 1, 130], [11, 60, 0]):
        q = rows(g, sum(new), H, d, dtype=dtype)
        out, _ = step(new, sum(new) + 5, lambda p: h.hippo_prefill_attention_paged(q, k_pool, v_pool, table, p[2], p[3]))
        lens_k = [len(x[0]) for x in held]
        ref = prefill_reference(q, torch.cat([cache(0, b) for b in range(B)]), torch.cat([cache(1, b) for b in range(B)]), new, lens_k)
        check(out[:sum(new)], ref[0], ref[1])
    n = 21
    for seed in (1, 2):
        parents = [some_tree(n, seed + b) for b in range(B)]
        q = rows(g, B, n, H, d, dtype=dtype)
        ctx, tree = lens.clone(), int32(parents)
        out, (k, v) = step([n] * B, n * B, lambda p: h.hippo_tree_attention_paged(q, k_pool, v_pool, table, tree, ctx))
        longest = max(len(x[0]) for x in held)
        caches = [torch.stack([torch.nn.functional.pad(cache(x, b), (0, 0, 0, 0, 0, longest - len(held[b][0]))) for b in range(B)])
                  .transpose(1, 2) for x in (0, 1)]
        ref = tree_reference(q, *caches, parents, ctx.tolist())
        check(out, ref[0], ref[1])
        # the paths to nodes 20, 7 and 0 are accepted: the trees' rows go back, the paths' rows are written again
        paths = []
        for b, node in enumerate((20, 7, 0)):
            path = []
            while node >= 0:
                path.append(node)
                node = parents[b][node]
            paths.append(path[::-1])
        p = h.hippo_plan_pages(lens, int32([-n] * B), table, free, n_free, page, 0)
        lens, n_free = p[3], p[4]
        kept = [len(x) for x in paths]
        p = h.hippo_plan_pages(lens, int32(kept), table, free, n_free, page, 64)
        lens, n_free = p[3], p[4]
        pick = [b * n + i for b, path in enumerate(paths) for i in path]
        h.hippo_write_kv_paged(k, v, p[0], k_pool, v_pool, rows=int32(pick + [-1] * (64 - len(pick))))
        for b in range(B):
            for x, rows_ in zip((0, 1), (k, v)):
                held[b][x] = held[b][x][:-n] + [rows_[b * n + i] for i in paths[b]]
    p = h.hippo_plan_pages(lens, -lens, table, free, n_free, page, 0)      # all done
    assert p[4].tolist() == [n_pool] and sorted(free.tolist()) == list(range(n_pool)) and p[3].tolist() == [0] * B
