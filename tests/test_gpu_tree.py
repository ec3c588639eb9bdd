"""GPU parity: hippo_tree_attention(_paged) against softmax in 64 bits, with the bounds that attention_reference.py derives."""
import pytest
import torch

from attention_reference import attend, check, check_lse
from test_gpu_prefill import TYPES, guarded_pools, pages_of, rows

pytestmark = pytest.mark.gpu


def seen(parents, ctx, total):
    """[n, total] truth values, node by node up the tree"""
    n = len(parents)
    sees = torch.zeros((n, total), dtype=torch.bool)
    for i in range(n):
        path, j = [], i
        while 0 <= j:
            path.append(j)
            if not -1 <= parents[j] < j:
                path = None
                break
            j = parents[j]
        if path is not None:
            sees[i, :ctx] = True
            sees[i, [ctx + j for j in path]] = True
    return sees.cuda()


def reference(q, k, v, parents, ctx, scale=None):
    """q [B, n, H, d], caches [B, Hkv, N, d], lists -> out, bound, lse and bound [B, H, n]"""
    B, n, H, d = q.shape
    G = H // k.shape[1]
    out, bound = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse, lse_bound = (torch.zeros((B, H, n), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        m = ctx[b] + n
        sees = seen(parents[b], ctx[b], m)
        for h in range(H):
            out[b, :, h], bound[b, :, h], lse[b, h], lse_bound[b, h] = attend(q[b, :, h], k[b, h // G, :m], v[b, h // G, :m], sees, scale)
    return out, bound, lse, lse_bound


def verify(got, ref, what=""):
    check(got[0], ref[0], ref[1], what)
    check_lse(got[1], ref[2], ref[3], what)


def some_tree(n, seed, padding=0):
    g = torch.Generator().manual_seed(seed)
    back = (torch.rand(n, generator=g) ** 2 * 9).long()
    parents = [max(-1, i - 1 - int(back[i])) for i in range(n)]
    return parents[:n - padding] + [-2] * padding


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(B, n, N, H, Hkv, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return rows(g, B, n, H, d, dtype=dtype), rows(g, B, Hkv, N, d, dtype=dtype), rows(g, B, Hkv, N, d, dtype=dtype)


@pytest.mark.parametrize("H,Hkv,d", [(4, 2, 64), (14, 2, 64), (28, 4, 128), (64, 8, 128), (3, 3, 64), (16, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,ctx", [(1, [0, 1]), (1, [700, 64]), (2, [63, 64]), (8, [832, 0]), (13, [65, 300]), (32, [31, 511]), (33, [1000, 7]),
                                   (64, [640, 129]), (64, [0, 2000])])
def test_trees(hippo, dtype, H, Hkv, d, n, ctx):
    q, k, v = make(2, n, max(ctx) + n + 3, H, Hkv, d, dtype, n)
    parents = [some_tree(n, 1), some_tree(n, 2, padding=n // 4)]
    got = hippo.hippo_tree_attention(q, k, v, int32(parents), int32(ctx), want_lse=True)
    verify(got, reference(q, k, v, parents, ctx), "%s %s" % (n, ctx))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("splits", [0, 1, 2, 7, 64])
def test_splits(hippo, dtype, splits):
    q, k, v = make(2, 20, 1520, 14, 2, 64, dtype, 5)
    parents = [some_tree(20, 3)] * 2
    got = hippo.hippo_tree_attention(q, k, v, int32(parents), int32([1500, 3]), num_splits=splits, want_lse=True)
    verify(got, reference(q, k, v, parents, [1500, 3]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,Hkv,d", [(2, 1, 64), (1, 1, 128), (14, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("n,first", [(64, 0), (64, 66), (37, 100)])
def test_a_tree_anywhere_in_a_stage(hippo, dtype, H, Hkv, d, n, first):
    """contexts of 66 lengths in a row, a last node that is none and whose rows of K and V are no numbers"""
    ctx = list(range(first, first + 66))
    q, k, v = make(66, n, max(ctx) + n, H, Hkv, d, dtype, first + n)
    parents = [some_tree(n, 10 + b, padding=1) for b in range(66)]
    clean_k, clean_v = k.clone(), v.clone()
    for b, c in enumerate(ctx):
        if b % 3:
            k[b, :, c + n - 1:] = float("nan")
            v[b, :, c + n - 1:] = float("nan") if b % 3 == 1 else float("inf")
    got = hippo.hippo_tree_attention(q, k, v, int32(parents), int32(ctx), want_lse=True)
    verify(got, reference(q, clean_k, clean_v, parents, ctx))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 6, 64])
def test_a_chain_is_a_verification(hippo, dtype, n):
    """a tree without branches sees what hippo_verify_attention's rows see"""
    q, k, v = make(2, n, 900 + n, 28, 4, 128, dtype, 6)
    chain = list(range(-1, n - 1))
    got = hippo.hippo_tree_attention(q, k, v, int32(chain), 900, want_lse=True)
    verify(got, reference(q, k, v, [chain] * 2, [900] * 2))
    want, _ = hippo.hippo_verify_attention(q, k, v, 900, want_lse=True)
    ref = reference(q, k, v, [chain] * 2, [900] * 2)
    assert ((got[0].double() - want.double()).abs() <= 3 * ref[1]).all()      # (its slices' outputs are rounded once more)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nodes_that_are_none(hippo, dtype):
    """parents below -1, at or behind the node, and descendants of such nodes: zeros, and nobody sees their rows"""
    n, ctx = 12, 100
    parents = [-1, 0, -2, 2, 4, 1, 9, 3, 2 ** 31 - 1, -(2 ** 31), 5, 11]
    q, k, v = make(1, n, ctx + n, 8, 2, 64, dtype, 7)
    ref = reference(q, k, v, [parents], [ctx])
    none = torch.tensor([i in (2, 3, 4, 6, 7, 8, 9, 11) for i in range(n)], device="cuda")
    for i in torch.nonzero(none)[:, 0].tolist():
        k[:, :, ctx + i], v[:, :, ctx + i] = float("nan"), float("inf")
    out, lse = hippo.hippo_tree_attention(q, k, v, int32([parents]), int32([ctx]), want_lse=True)
    verify((out, lse), ref)
    assert (out[:, none] == 0).all() and (lse[:, :, none] == -float("inf")).all()
    every = hippo.hippo_tree_attention(q, k, v, int32([[-2] * n]), int32([ctx]))
    assert (every == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("poison", [float("nan"), float("inf")])
def test_siblings_do_not_reach_each_other(hippo, dtype, poison):
    parents, ctx = [-1, 0, 0, 1, 2, -1], 70
    q, k, v = make(1, 6, ctx + 6 + 20, 8, 2, 64, dtype, 8)
    ref = reference(q, k, v, [parents], [ctx])
    k[:, :, ctx + 2], v[:, :, ctx + 2] = poison, poison            # node 2: seen by itself and node 4
    k[:, :, ctx + 6:], v[:, :, ctx + 6:] = poison, poison          # behind the tree
    out, lse = hippo.hippo_tree_attention(q, k, v, int32(parents), int32([ctx]), want_lse=True)
    keep = torch.tensor([0, 1, 3, 5], device="cuda")
    check(out[:, keep], ref[0][:, keep], ref[1][:, keep])
    check_lse(lse[:, :, keep], ref[2][:, :, keep], ref[3][:, :, keep])


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (8, 2, 128)), ("fp32", (4, 2, 64))])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("splits", [0, 3])
def test_paged(hippo, dtype, heads, page, splits):
    H, Hkv, d = heads
    n, ctx = 17, [800, 0, 65, 2000]
    g = torch.Generator(device="cuda").manual_seed(9)
    lens = [c + n for c in ctx]
    q = rows(g, 4, n, H, d, dtype=dtype)
    k, v = (rows(g, sum(lens), Hkv, d, dtype=dtype) for _ in range(2))
    k_pool, v_pool, table = pages_of(g, k, v, lens, page)
    caches = []
    for x in (k, v):
        c = torch.zeros((4, Hkv, max(lens), d), dtype=x.dtype, device="cuda")
        for b, part in enumerate(torch.split(x, lens)):
            c[b, :, :lens[b]] = part.transpose(0, 1)
        caches.append(c)
    parents = [some_tree(n, b, padding=b) for b in range(4)]
    got = hippo.hippo_tree_attention_paged(q, k_pool, v_pool, table, int32(parents), int32(ctx), num_splits=splits, want_lse=True)
    verify(got, reference(q, *caches, parents, ctx))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides(hippo, dtype):
    """a cache of interleaved heads, parents of every second row, a query and an output in place of others"""
    g = torch.Generator(device="cuda").manual_seed(10)
    B, n, H, Hkv, d, ctx = 3, 9, 8, 2, 64, [50, 120, 7]
    k, v = (rows(g, B, 140, Hkv, d, dtype=dtype).transpose(1, 2) for _ in range(2))
    q = rows(g, B, n, H, d, dtype=dtype)
    parents = [some_tree(n, b) for b in range(B)]
    wide = torch.full((2 * B, n + 7), -9, dtype=torch.int32, device="cuda")
    wide[::2, :n] = int32(parents)
    out = torch.empty_like(q)
    hippo.hippo_tree_attention(q, k, v, wide[::2, :n], int32(ctx), out=out)
    ref = reference(q, k, v, parents, ctx)
    check(out, ref[0], ref[1])


def test_lengths_outside_the_cache_are_cut_off(hippo):
    q, k, v = make(2, 4, 60, 4, 2, 64, "bf16", 11)
    parents = [[-1, 0, 1, 0]] * 2
    got = hippo.hippo_tree_attention(q, k, v, int32(parents), int32([-9, 2 ** 31 - 1]))
    ref = reference(q, k, v, parents, [0, 56])
    check(got, ref[0], ref[1])


def test_streams_and_graphs(hippo):
    """two graphs with a workspace and outputs of their own; lengths and trees are read by the replays"""
    q, k, v = make(2, 10, 700, 28, 4, 128, "bf16", 12)
    trees = [[some_tree(10, s), some_tree(10, s + 1, padding=2)] for s in (1, 5, 9)]
    lengths = [[690, 12], [0, 333], [64, 689]]
    parents, ctx = int32(trees[0]), int32(lengths[0])
    want = hippo.hippo_tree_attention(q, k, v, parents, ctx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hippo.hippo_tree_attention(q, k, v, parents, ctx, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graphs, outs = [], []
    for splits in (1, 4):
        out = torch.zeros_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hippo.hippo_tree_attention(q, k, v, parents, ctx, num_splits=splits, out=out)
        graphs.append(graph)
        outs.append(out)
    for tree, lens in zip(trees, lengths):
        parents.copy_(int32(tree))
        ctx.copy_(int32([min(x, 690) for x in lens]))
        for out, graph in zip(outs, graphs):
            out.zero_()
            graph.replay()
        ref = reference(q, k, v, tree, [min(x, 690) for x in lens])
        for out in outs:
            check(out, ref[0], ref[1])
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,heads,n,ctx", [("bf16", (28, 4, 128), 16, [16640]), ("bf16", (64, 8, 128), 64, [9000, 300, 20000]),
                                               ("bf16", (14, 2, 64), 48, [33280]), ("fp32", (28, 4, 128), 64, [9999])])
def test_long_caches(hippo, dtype, heads, n, ctx):
    H, Hkv, d = heads
    q, k, v = make(len(ctx), n, max(ctx) + n, H, Hkv, d, dtype, 13)
    parents = [some_tree(n, b, padding=b) for b in range(len(ctx))]
    verify(hippo.hippo_tree_attention(q, k, v, int32(parents), int32(ctx), want_lse=True), reference(q, k, v, parents, ctx))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,n,longest", [(2, 5, 3000), (3, 64, 900), (17, 9, 700), (64, 3, 500), (65, 3, 500), (130, 1, 200)])
def test_batches_of_very_different_lengths(hippo, dtype, B, n, longest):
    """blocks are dealt out by length to 2 to 64 sequences, evenly to more"""
    g = torch.Generator().manual_seed(B)
    ctx = [int(longest * float(x) ** 3) for x in torch.rand(B, generator=g)]
    ctx[0], ctx[-1] = 0, longest
    q, k, v = make(B, n, longest + n, 4, 2, 64, dtype, 14)
    parents = [some_tree(n, b, padding=b % max(1, n // 2)) for b in range(B)]
    want = reference(q, k, v, parents, ctx)
    for splits in (0, 2, 5, 64):
        got = hippo.hippo_tree_attention(q, k, v, int32(parents), int32(ctx), num_splits=splits, want_lse=True)
        verify(got, want, "%d sequences, %d splits" % (B, splits))


def test_one_length_for_all_needs_no_tensor(hippo):
    q, k, v = make(3, 7, 500, 14, 2, 64, "bf16", 15)
    parents = some_tree(7, 1)
    a = hippo.hippo_tree_attention(q, k, v, int32(parents), 400)
    b = hippo.hippo_tree_attention(q, k, v, int32([parents] * 3), int32([400] * 3), num_splits=1)
    ref = reference(q, k, v, [parents] * 3, [400] * 3)
    check(a, ref[0], ref[1])
    check(b, ref[0], ref[1])


def test_more_than_two_million_blocks(hippo):
    """65535 trees of one node without a context, 33 heads: its row of V is the output, bit for bit"""
    q, k, v = make(65535, 1, 1, 33, 33, 64, "bf16", 16)
    assert torch.equal(hippo.hippo_tree_attention(q, k, v, int32([-1]), 0)[:, 0], v[:, :, 0])


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (8, 2, 128)), ("fp32", (4, 2, 64))])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("splits", [1, 3])
def test_numbers_that_are_no_pages_are_taken_for_the_pool_s_ends(hippo, dtype, heads, page, splits):
    H, Hkv, d = heads
    g = torch.Generator(device="cuda").manual_seed(17)
    (k_pool, v_pool), table, taken = guarded_pools(g, 5, page, Hkv, d, dtype)
    n, ctx = 11, [6 * page - 11, 5 * page - 10]
    q = rows(g, 2, n, H, d, dtype=dtype)
    parents = [some_tree(n, b, padding=b) for b in range(2)]
    got = hippo.hippo_tree_attention_paged(q, k_pool, v_pool, int32(table), int32(parents), int32(ctx), num_splits=splits, want_lse=True)
    k, v = (torch.stack([x[t].flatten(0, 1).transpose(0, 1) for t in taken]) for x in (k_pool, v_pool))
    verify(got, reference(q, k, v, parents, ctx))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B", [1, 3, 65])
def test_a_cache_with_much_more_room_than_rows(hippo, dtype, B):
    """over pages, with a table of 131072 rows: one tree, a batch dealt by length, one dealt evenly"""
    n, ctx = 6, [(37 * b) % 150 for b in range(B)]
    q, k, v = make(B, n, max(ctx) + n, 4, 2, 64, dtype, 18)
    lens = [c + n for c in ctx]
    g = torch.Generator(device="cuda").manual_seed(19)
    packed = [torch.cat([x[b, :, :m].transpose(0, 1) for b, m in enumerate(lens)]) for x in (k, v)]
    k_pool, v_pool, table = pages_of(g, *packed, lens, 16)
    wide = torch.full((B, 8192), -9, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    parents = [some_tree(n, b, padding=b % 3) for b in range(B)]
    want = reference(q, k, v, parents, ctx)
    for splits in (0, 1, 64):
        got = hippo.hippo_tree_attention_paged(q, k_pool, v_pool, wide, int32(parents), int32(ctx), num_splits=splits, want_lse=True)
        verify(got, want, "%d splits" % splits)
