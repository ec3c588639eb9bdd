"""GPU parity: hippo_prefill_attention(_paged) against softmax in 64 bits, with the bounds that attention_reference.py derives."""
import itertools

import numpy as np
import pytest
import torch

from attention_reference import attend, check, check_lse

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def rows(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(TYPES[dtype])


def offsets(lens):
    return torch.tensor([0] + list(itertools.accumulate(lens)), dtype=torch.int32, device="cuda")


def make(lens_q, lens_k, H, Hkv, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = rows(g, sum(lens_q), H, d, dtype=dtype)
    k, v = (rows(g, sum(lens_k), Hkv, d, dtype=dtype) for _ in range(2))
    return q, k, v


def reference(q, k, v, lens_q, lens_k, scale=None):
    """out, bound [T, H, d], lse and bound [H, T]"""
    T, H, d = q.shape
    G = H // k.shape[1]
    out, bound = (torch.zeros((T, H, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, lse_bound = (torch.zeros((H, T), dtype=torch.float64, device="cuda") for _ in range(2))
    a = b = 0
    for n, m in zip(lens_q, lens_k):
        sees = torch.arange(m, device="cuda") <= m - n + torch.arange(n, device="cuda")[:, None]
        for h in range(H):
            o = attend(q[a:a + n, h], k[b:b + m, h // G], v[b:b + m, h // G], sees, scale)
            out[a:a + n, h], bound[a:a + n, h], lse[h, a:a + n], lse_bound[h, a:a + n] = o
        a, b = a + n, b + m
    return out, bound, lse, lse_bound


def verify(got, ref, what=""):
    check(got[0], ref[0], ref[1], what)
    check_lse(got[1], ref[2], ref[3], what)


LENS = [[1], [2], [31], [32], [33], [64], [65], [127], [200], [257], [600], [1, 1], [37, 1, 64, 0, 5], [0, 0, 3], [63, 64, 65, 66], [300, 7, 150, 520]]


@pytest.mark.parametrize("H,Hkv,d", [(4, 2, 64), (14, 2, 64), (28, 4, 128), (3, 3, 128), (16, 1, 64), (8, 8, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_whole_prompts(hippo, dtype, H, Hkv, d):
    for i, lens in enumerate(LENS):
        q, k, v = make(lens, lens, H, Hkv, d, dtype, i)
        got = hippo.hippo_prefill_attention(q, k, v, offsets(lens), want_lse=True)
        verify(got, reference(q, k, v, lens, lens), "%s %s" % (dtype, lens))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens_q,lens_k", [([1], [1000]), ([1, 1, 1], [1, 64, 65]), ([17], [2000]), ([5, 100, 0, 33], [700, 100, 40, 34]),
                                           ([9, 4], [3, 4]), ([300], [0]), ([70, 2], [0, 2]), ([256], [4224])])
@pytest.mark.parametrize("splits", [0, 1, 3, 64])
def test_pieces_behind_longer_keys(hippo, dtype, lens_q, lens_k, splits):
    """rows that see nothing (more queries than keys) among them"""
    q, k, v = make(lens_q, lens_k, 14, 2, 64, dtype, 3)
    got = hippo.hippo_prefill_attention(q, k, v, offsets(lens_q), offsets(lens_k), num_splits=splits, want_lse=True)
    verify(got, reference(q, k, v, lens_q, lens_k), "%s %s" % (lens_q, lens_k))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(hippo, dtype):
    """more sequences than a wave has lanes"""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 40, 150)]
    lens_k = [n + int(x) for n, x in zip(lens, rng.integers(0, 90, 150))]
    q, k, v = make(lens, lens_k, 4, 2, 64, dtype, 6)
    verify(hippo.hippo_prefill_attention(q, k, v, offsets(lens), offsets(lens_k), want_lse=True), reference(q, k, v, lens, lens_k))


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (4, 2, 64)), ("fp32", (8, 2, 128))])
@pytest.mark.parametrize("lens", [[5000], [2600, 1, 1900, 300]])
def test_long_prompts(hippo, dtype, heads, lens):
    """tiles of every size, the largest ones among them"""
    H, Hkv, d = heads
    q, k, v = make(lens, lens, H, Hkv, d, dtype, 7)
    verify(hippo.hippo_prefill_attention(q, k, v, offsets(lens), want_lse=True), reference(q, k, v, lens, lens))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slices_of_a_fused_projection(hippo, dtype):
    H, Hkv, d, lens = 14, 2, 64, [100, 33]
    g = torch.Generator(device="cuda").manual_seed(8)
    fused = rows(g, sum(lens), H + 2 * Hkv, d, dtype=dtype)
    q, k, v = fused[:, :H], fused[:, H:H + Hkv], fused[:, H + Hkv:]
    got = hippo.hippo_prefill_attention(q, k, v, offsets(lens), want_lse=True)
    verify(got, reference(q, k, v, lens, lens))
    heads_first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    again = hippo.hippo_prefill_attention(*heads_first, offsets(lens), want_lse=True)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sharp", [0.0, 30.0])
def test_scales(hippo, dtype, sharp):
    """equal logits, and logits of which one has all the weight"""
    q, k, v = make([150], [150], 4, 2, 64, dtype, 9)
    if sharp == 0.0:
        q = torch.zeros_like(q)
    scale = sharp / 8 or None
    got = hippo.hippo_prefill_attention(q, k, v, offsets([150]), softmax_scale=scale or 0.0, want_lse=True)
    verify(got, reference(q, k, v, [150], [150], scale))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("splits", [0, 2])
def test_what_a_row_does_not_see_does_not_reach_it(hippo, dtype, poison, splits):
    lens_q, lens_k = [100, 90], [190, 90]
    q, k, v = make(lens_q, lens_k, 8, 2, 128 if dtype == "bf16" else 64, dtype, 10)
    ref = reference(q, k, v, lens_q, lens_k)
    k, v = k.clone(), v.clone()
    k[190 - 30:190], v[190 - 30:190, :, 5:] = poison, poison        # the last 30 rows of sequence 0: seen by its last 30 query rows
    k[-1], v[-1] = poison, poison                                    # sequence 1's last row
    out, lse = hippo.hippo_prefill_attention(q, k, v, offsets(lens_q), offsets(lens_k), num_splits=splits, want_lse=True)
    clean = torch.ones(190, dtype=torch.bool, device="cuda")
    clean[70:100] = False
    clean[-1] = False
    check(out[clean], ref[0][clean], ref[1][clean])
    check_lse(lse[:, clean], ref[2][:, clean], ref[3][:, clean])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_values_that_are_seen(hippo, dtype):
    """an infinity of V reaches the rows that see it, as an infinity, and no other row or channel"""
    q, k, v = make([70], [70], 4, 2, 64, dtype, 11)
    ref = reference(q, k, v, [70], [70])
    v = v.clone()
    v[40, 0, 7], v[50, 1, 9], v[60, 1, 11] = float("inf"), -float("inf"), float("nan")
    out = hippo.hippo_prefill_attention(q, k, v, offsets([70])).float()
    assert (out[40:, :2, 7] == float("inf")).all() and (out[50:, 2:, 9] == -float("inf")).all() and torch.isnan(out[60:, 2:, 11]).all()
    out[40:, :2, 7], out[50:, 2:, 9], out[60:, 2:, 11] = (ref[0][40:, :2, 7].float(), ref[0][50:, 2:, 9].float(), ref[0][60:, 2:, 11].float())
    check(out, ref[0], ref[1] + 1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("splits", [0, 1, 2, 4, 31])
@pytest.mark.parametrize("low", [-400.0, -float("inf")])
def test_infinite_values_of_no_weight_are_seen_however_the_keys_are_split(hippo, dtype, splits, low):
    """the first 700 of 2000 keys get weights of exp(-1000) and less, 0 in fp32: 0 times infinity is no number, in whichever part it comes about"""
    q, k, v = make([17], [2000], 4, 2, 64, dtype, 22)
    q[..., 0], k[..., 0], k[:700, :, 0] = 20, 0, low
    v[5, 0, 7], v[300, 1, 9], v[600, 1, 11] = float("inf"), -float("inf"), float("nan")
    out = hippo.hippo_prefill_attention(q, k, v, offsets([17]), offsets([2000]), num_splits=splits).float()
    finite = torch.ones_like(out, dtype=torch.bool)
    finite[:, :2, 7] = finite[:, 2:, 9] = finite[:, 2:, 11] = False
    assert bool((torch.isfinite(out) == finite).all())
    v[5, 0, 7] = v[300, 1, 9] = v[600, 1, 11] = 0
    ref = reference(q, k[700:], v[700:], [17], [1300])
    check(out[finite], ref[0][finite], ref[1][finite])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("splits", [1, 4])
def test_rows_of_no_sequence_stay(hippo, dtype, splits):
    lens = [40, 3, 100]
    q, k, v = make([10] + lens + [20], [10] + lens + [20], 4, 2, 64, dtype, 12)
    cu = offsets([10] + lens)[1:].contiguous()
    out = torch.full_like(q, 7.0)
    got = hippo.hippo_prefill_attention(q, k, v, cu, num_splits=splits, out=out)
    assert got is out or got.data_ptr() == out.data_ptr()
    assert (out[:10] == 7).all() and (out[-20:] == 7).all()
    ref = reference(q[10:-20], k[10:-20], v[10:-20], lens, lens)
    check(out[10:-20], ref[0], ref[1])


def test_offsets_outside_the_buffers_are_cut_off(hippo):
    q, k, v = make([50], [50], 4, 2, 64, "bf16", 13)
    cu = torch.tensor([-5, 20, 10, 1000, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    guard = torch.full((50 + 200, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    hippo.hippo_prefill_attention(q, k, v, cu, out=guard[:50])
    assert (guard[50:] == 7).all()


def pages_of(g, k, v, lens, page, spare=3, dtype=torch.int32):
    """pools with the sequences' rows on pages in random order, the rest poisoned, and the table"""
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(dtype)
    k_pool, v_pool = (torch.full((total, page) + x.shape[1:], float("nan"), dtype=x.dtype, device="cuda") for x in (k, v))
    table = torch.full((len(lens), max(need + [1]) + 2), -1, dtype=dtype, device="cuda")
    at = row = 0
    for b, n in enumerate(lens):
        for i in range(need[b]):
            pg = int(order[at])
            table[b, i] = pg
            m = min(page, n - i * page)
            k_pool[pg, :m], v_pool[pg, :m] = k[row + i * page:row + i * page + m], v[row + i * page:row + i * page + m]
            at += 1
        row += n
    return k_pool, v_pool, table


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (8, 2, 128)), ("fp32", (4, 2, 64))])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("splits", [0, 5])
def test_paged(hippo, dtype, heads, page, splits):
    """whatever the pages hold behind a sequence's last row"""
    H, Hkv, d = heads
    lens_q, lens_k = [60, 1, 0, 129, 16], [800, 65, 30, 129, 16]
    q, k, v = make(lens_q, lens_k, H, Hkv, d, dtype, 14)
    g = torch.Generator(device="cuda").manual_seed(15)
    k_pool, v_pool, table = pages_of(g, k, v, lens_k, page)
    lens = torch.tensor(lens_k, dtype=torch.int32, device="cuda")
    got = hippo.hippo_prefill_attention_paged(q, k_pool, v_pool, table, offsets(lens_q), lens, num_splits=splits, want_lse=True)
    verify(got, reference(q, k, v, lens_q, lens_k))


def test_pages_outside_the_pool(hippo):
    """a table with numbers that are no pages: any result, no access outside"""
    q, k, v = make([64], [64], 4, 2, 64, "bf16", 16)
    table = torch.tensor([[-7, 2 ** 31 - 1, 5, 12]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out = hippo.hippo_prefill_attention_paged(q, k.view(4, 16, 2, 64), v.view(4, 16, 2, 64), table, offsets([64]), lens)
    torch.cuda.synchronize()
    assert out.shape == q.shape


def test_a_pool_beyond_32_bit_offsets(hippo):
    """pages further apart than 2^32 bytes"""
    page, Hkv, d = 16, 2, 64
    g = torch.Generator(device="cuda").manual_seed(17)
    k, v = (rows(g, 40, Hkv, d, dtype="bf16") for _ in range(2))
    q = rows(g, 40, 4, d, dtype="bf16")
    wide = torch.empty((70000 * 16, page, Hkv, d), dtype=torch.bfloat16, device="cuda")       # 4.6 GB
    table = torch.tensor([[70000 * 16 - 1, 3, 70000 * 15]], dtype=torch.int32, device="cuda")
    for i, pg in enumerate(table[0].tolist()):
        m = min(16, 40 - 16 * i)
        wide[pg, :m] = k[16 * i:16 * i + m]
    wide_v = torch.empty_like(wide)
    for i, pg in enumerate(table[0].tolist()):
        m = min(16, 40 - 16 * i)
        wide_v[pg, :m] = v[16 * i:16 * i + m]
    lens = torch.tensor([40], dtype=torch.int32, device="cuda")
    got = hippo.hippo_prefill_attention_paged(q, wide, wide_v, table, offsets([40]), lens, want_lse=True)
    verify(got, reference(q, k, v, [40], [40]))


def test_streams_and_graphs(hippo):
    lens = [130, 1, 77]
    q, k, v = make(lens, lens, 14, 2, 64, "bf16", 18)
    cu = offsets(lens)
    want = hippo.hippo_prefill_attention(q, k, v, cu, num_splits=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hippo.hippo_prefill_attention(q, k, v, cu, num_splits=3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hippo.hippo_prefill_attention(q, k, v, cu, num_splits=3, out=out)
    for lens in ([130, 1, 77], [8, 0, 200], [200, 8, 0]):            # the lengths are read by the replay
        cu.copy_(offsets(lens))
        out.zero_()
        graph.replay()
        ref = reference(q[:sum(lens)], k[:sum(lens)], v[:sum(lens)], lens, lens)
        check(out[:sum(lens)], ref[0], ref[1], str(lens))
        torch.cuda.synchronize()


def test_the_same_bits_every_time(hippo):
    lens = [700, 300]
    q, k, v = make(lens, lens, 28, 4, 128, "bf16", 19)
    first = hippo.hippo_prefill_attention(q, k, v, offsets(lens))
    for _ in range(5):
        assert torch.equal(hippo.hippo_prefill_attention(q, k, v, offsets(lens)), first)


def test_no_rows(hippo):
    q, k, v = make([0], [0], 4, 2, 64, "bf16", 20)
    assert hippo.hippo_prefill_attention(q, k, v, offsets([0])).shape == (0, 4, 64)
    q, k, v = make([5], [0], 4, 2, 64, "fp32", 21)
    out, lse = hippo.hippo_prefill_attention(q, k, v, offsets([5]), offsets([0]), want_lse=True)
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("dtype,heads,blocks", [("bf16", (28, 4, 128), {2, 4}), ("bf16", (14, 2, 64), {1, 2, 4}), ("fp32", (4, 2, 64), {1, 2, 4}),
                                                ("fp32", (28, 4, 128), {2, 4})])
def test_every_tile_size(hippo, kernels, dtype, heads, blocks):
    """few and many rows, so that each size of a block is taken, over lengths that end around its stages: none, one and several that need
    no mask"""
    H, Hkv, d = heads
    sizes = set()
    some = [1, 20, 31, 64, 65, 127, 128, 129, 191, 192, 256, 257, 320, 321, 385, 449, 513, 640]
    for seqs, lens_of in ((1, some), (8, some), (24, some[7:]), (60, [64, 129, 257, 385])):
        for n in lens_of:
            if dtype == "fp32" and (d == 128 and n * seqs > 4000):
                continue
            lens = [n] * seqs
            q, k, v = make(lens, lens, H, Hkv, d, dtype, n)
            cu = offsets(lens)
            call = lambda: hippo.hippo_prefill_attention(q, k, v, cu, want_lse=True)      # noqa: E731
            out, lse = call()
            # row blocks and token groups of a block; one group of four: two such blocks on a compute unit
            sizes |= {tuple(int(x) for x in name.split("attn_rows")[1].split("ELi")[1:3]) for name in kernels(call) if "attn_rows" in name}
            first, last = slice(0, n), slice((seqs - 1) * n, seqs * n)
            for at in (first, last):
                ref = reference(q[at], k[at], v[at], [n], [n])
                check(out[at], ref[0], ref[1], "%d x %d" % (seqs, n))
                check_lse(lse[:, at], ref[2], ref[3], "%d x %d" % (seqs, n))
            # equal rows of other sequences: the same bits from another place in the launch
            if seqs > 2:
                q2, k2, v2 = (torch.cat([x[first], x[n:-n], x[first]]) for x in (q, k, v))
                again = hippo.hippo_prefill_attention(q2, k2, v2, cu)
                assert torch.equal(again[first], again[last])
    assert {rb for rb, _ in sizes} >= blocks, sizes
    assert ((4, 1) in sizes) == (heads[2] == 64 or dtype == "bf16"), sizes


def test_few_rows_over_longer_keys(hippo, kernels):
    q, k, v = make([64], [364], 64, 8, 128, "bf16", 62)
    cu_q, cu_k = offsets([64]), offsets([364])
    call = lambda: hippo.hippo_prefill_attention(q, k, v, cu_q, cu_k, want_lse=True)      # noqa: E731
    verify(call(), reference(q, k, v, [64], [364]))
    assert {name.split("attn_rows")[1].split("ELi")[1] for name in kernels(call) if "attn_rows" in name} == {"1"}


@pytest.mark.parametrize("dtype,heads,lens,block", [
    ("bf16", (28, 4, 128), [4200], (8, 1)), ("bf16", (14, 2, 64), [8191], (8, 1)), ("fp32", (28, 4, 128), [700] * 8, (8, 1)),
    ("bf16", (28, 4, 128), [2049], (4, 2)), ("bf16", (14, 2, 64), [4500], (4, 2)), ("fp32", (28, 4, 64), [2500], (4, 2)),
    ("bf16", (14, 2, 64), [1500] * 9, (4, 1)), ("bf16", (28, 4, 128), [511] * 60, (4, 1)), ("fp32", (8, 2, 64), [900] * 40, (4, 1))])
def test_longer_prompts_of_every_block(hippo, kernels, dtype, heads, lens, block):
    """row blocks and token groups of a block, see above"""
    H, Hkv, d = heads
    q, k, v = make(lens, lens, H, Hkv, d, dtype, 61)
    cu = offsets(lens)
    call = lambda: hippo.hippo_prefill_attention(q, k, v, cu, want_lse=True)              # noqa: E731
    out, lse = call()
    assert {tuple(int(x) for x in name.split("attn_rows")[1].split("ELi")[1:3]) for name in kernels(call) if "attn_rows" in name} == {block}
    # rows at both ends and around the middle of the last sequence, each as the last row of a shorter one
    start, n = sum(lens[:-1]), lens[-1]
    for i in (0, 1, 255, n // 2, n // 2 + 37, n - 2, n - 1):
        at, upto = slice(start + i, start + i + 1), slice(start, start + i + 1)
        ref = reference(q[at], k[upto], v[upto], [1], [i + 1])
        check(out[at], ref[0], ref[1], i)
        check_lse(lse[:, at], ref[2], ref[3], i)


def test_two_calls_at_once(hippo):
    """on streams of their own, each with its own workspace"""
    lens = [400, 90]
    a, b = make(lens, lens, 28, 4, 128, "bf16", 30), make(lens, lens, 28, 4, 128, "bf16", 31)
    cu = offsets(lens)
    want = [hippo.hippo_prefill_attention(*x, cu, num_splits=4) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[hippo.hippo_prefill_attention(*x, cu, num_splits=4, stream=s) for _ in range(5)] for x, s in zip((a, b), streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for gs, w in zip(got, want) for g in gs)


def test_more_than_two_million_blocks(hippo):
    """8300 sequences of one row, 256 heads: a row's only key has all the weight, and its row of V is the output, bit for bit"""
    g = torch.Generator(device="cuda").manual_seed(63)
    q, k, v = (rows(g, 8300, 256, 64, dtype="bf16") for _ in range(3))
    out = hippo.hippo_prefill_attention(q, k, v, torch.arange(8301, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("splits", [0, 9, 64])
def test_a_long_sequence_beside_short_ones(hippo, dtype, splits):
    """the caller's number of blocks a tile, though most of the sequences have no stage for them"""
    lens_q, lens_k = [110, 5, 329, 11], [128, 5, 912, 20011]
    q, k, v = make(lens_q, lens_k, 4, 2, 64, dtype, 64)
    got = hippo.hippo_prefill_attention(q, k, v, offsets(lens_q), offsets(lens_k), num_splits=splits, want_lse=True)
    verify(got, reference(q, k, v, lens_q, lens_k))


def guarded_pools(g, n_pool, page, Hkv, d, dtype):
    """pools in the middle of larger buffers whose other pages hold no numbers, and a table of pages and of numbers just past either end of
    the pool with the pages that those are taken for"""
    pools = []
    for _ in range(2):
        whole = torch.full((n_pool + 16, page, Hkv, d), float("nan"), dtype=TYPES[dtype], device="cuda")
        whole[8:-8] = rows(g, n_pool, page, Hkv, d, dtype=dtype)
        pools.append(whole[8:-8])
    table = [[2, -1, n_pool, 1, n_pool + 7, 3], [-8, n_pool - 1, 0, n_pool + 1, -2, 2]]
    return pools, table, [[min(max(x, 0), n_pool - 1) for x in t] for t in table]


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (8, 2, 128)), ("fp32", (4, 2, 64))])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("splits", [1, 3])
def test_numbers_that_are_no_pages_are_taken_for_the_pool_s_ends(hippo, dtype, heads, page, splits):
    H, Hkv, d = heads
    g = torch.Generator(device="cuda").manual_seed(65)
    (k_pool, v_pool), table, taken = guarded_pools(g, 5, page, Hkv, d, dtype)
    lens_q, lens_k = [40, 3], [6 * page - 5, 5 * page + 1]
    q = rows(g, 43, H, d, dtype=dtype)
    got = hippo.hippo_prefill_attention_paged(q, k_pool, v_pool, torch.tensor(table, dtype=torch.int32, device="cuda"), offsets(lens_q),
                                              torch.tensor(lens_k, dtype=torch.int32, device="cuda"), num_splits=splits, want_lse=True)
    k, v = (torch.cat([x[t].flatten(0, 1)[:n] for t, n in zip(taken, lens_k)]) for x in (k_pool, v_pool))
    verify(got, reference(q, k, v, lens_q, lens_k))


@pytest.mark.parametrize("dtype,heads", [("bf16", (28, 4, 128)), ("bf16", (14, 2, 64)), ("fp32", (8, 2, 128)), ("fp32", (4, 2, 64))])
@pytest.mark.parametrize("lens_q,lens_k", [([1], [1]), ([300], [300]), ([90, 0, 7], [90, 40, 700])])
def test_a_table_much_wider_than_the_lengths(hippo, dtype, heads, lens_q, lens_k):
    """room for 131072 rows a sequence: most of the blocks that share a tile have no stage; what the unused columns hold is not looked at"""
    H, Hkv, d = heads
    q, k, v = make(lens_q, lens_k, H, Hkv, d, dtype, 66)
    g = torch.Generator(device="cuda").manual_seed(67)
    k_pool, v_pool, table = pages_of(g, k, v, lens_k, 16)
    wide = torch.full((len(lens_k), 8192), -9, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    lens = torch.tensor(lens_k, dtype=torch.int32, device="cuda")
    for splits in (0, 1, 64):
        got = hippo.hippo_prefill_attention_paged(q, k_pool, v_pool, wide, offsets(lens_q), lens, num_splits=splits, want_lse=True)
        verify(got, reference(q, k, v, lens_q, lens_k), "%d splits" % splits)
