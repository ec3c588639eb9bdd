"""GPU: hippo_evict_kv against a sort by (mass, row) on the host.  Rows and indices are copies and whole numbers: equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}


def kept_rows(mass, keep, first, recent):
    """[B, Hkv, N] -> [B, Hkv, keep]; NaN below every number, equal ones by the lower row"""
    B, Hkv, N = mass.shape
    x = mass.astype(np.float64)
    rank = np.where(np.isnan(x), np.inf, -x)
    isnan = np.isnan(x)
    out = np.empty((B, Hkv, keep), np.int64)
    k, last = keep - first - recent, N - recent
    for b in range(B):
        for h in range(Hkv):
            at = np.arange(first, last)
            order = at[np.lexsort((at, rank[b, h, at], isnan[b, h, at]))][:k]
            out[b, h] = np.concatenate([np.arange(first), np.sort(order), np.arange(last, N)])
    return out


def make(B, Hkv, N, d, dtype, seed, kind="heavy"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "heavy":
        mass = torch.exp(2 * torch.randn((B, Hkv, N), generator=g, device="cuda"))
        mass *= torch.rand((B, Hkv, N), generator=g, device="cuda") > 0.1
    elif kind == "ties":
        mass = torch.randint(0, 4, (B, Hkv, N), generator=g, device="cuda").float()
    elif kind == "equal":
        mass = torch.zeros((B, Hkv, N), device="cuda")
    else:                                                         # what a sum should not become, and signs of zero
        mass = torch.randn((B, Hkv, N), generator=g, device="cuda")
        pick = torch.randint(0, 6, (B, Hkv, N), generator=g, device="cuda")
        for i, v in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0)):
            mass[pick == i] = v
    if dtype == "fp8":
        k, v = (torch.randint(0, 256, (B, Hkv, N, d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    else:
        k, v = (torch.randn((B, Hkv, N, d), generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    return mass, k, v


def check(got, mass, k, v, keep, first, recent, what=""):
    idx, kd, vd, md = got
    want = kept_rows(mass.cpu().numpy(), keep, first, recent)
    np.testing.assert_array_equal(idx.cpu().numpy(), want, err_msg=str(what))
    at = torch.from_numpy(want).cuda()
    rows = at[..., None].expand(*at.shape, k.shape[3])
    assert torch.equal(kd[:, :, :keep].view(torch.uint8), torch.gather(k, 2, rows).view(torch.uint8)), what
    assert torch.equal(vd[:, :, :keep].view(torch.uint8), torch.gather(v, 2, rows).view(torch.uint8)), what
    assert torch.equal(md[:, :, :keep].contiguous().view(torch.int32), torch.gather(mass, 2, at).view(torch.int32)), what


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("fp32", 128), ("bf16", 64), ("bf16", 128), ("fp8", 64), ("fp8", 128)])
@pytest.mark.parametrize("B,Hkv,N,keep,first,recent", [
    (1, 1, 1, 1, 0, 0),             # the only row
    (1, 2, 1, 1, 1, 0),             # ... as the first, with nothing between
    (2, 3, 2, 1, 0, 1),             # only the recent
    (2, 2, 7, 7, 2, 3),             # all of them
    (1, 3, 65, 64, 0, 0),           # one row goes
    (3, 2, 300, 17, 4, 5),
    (2, 2, 1000, 20, 8, 12),        # nothing between is kept: first and recent rows alone
    (1, 2, 2049, 1024, 4, 64),      # size classes of the selection, and a row more
    (2, 4, 4100, 2000, 4, 1),
    (1, 2, 8193, 8192, 0, 1),
])
def test_rows_that_stay(hippo, dtype, d, B, Hkv, N, keep, first, recent):
    for kind in ("heavy", "ties"):
        mass, k, v = make(B, Hkv, N, d, dtype, N + keep, kind)
        got = hippo.hippo_evict_kv(mass, keep, k, v, n_first=first, n_recent=recent)
        check(got, mass, k, v, keep, first, recent, (dtype, kind))


@pytest.mark.parametrize("N", [8192 + 1, 12288, 12288 + 1, 20480, 20480 + 1, 32768, 32768 + 1, 36864, 36864 + 1, 57344, 57344 + 1])
@pytest.mark.parametrize("kind", ["heavy", "ties", "odd"])
def test_edges_of_the_classes(hippo, N, kind):
    """rows between as many as a class of keys a thread holds, and one more; indices and mass alone and with rows"""
    mass, k, v = make(1, 2, N + 3, 64, "fp8", N, kind)
    for keep in (5 + N // 7, N - 1):
        got = hippo.hippo_evict_kv(mass, keep, k, v, n_first=1, n_recent=2)
        check(got, mass, k, v, keep, 1, 2, keep)
        idx, none, none_too, md = hippo.hippo_evict_kv(mass, keep, None, None, n_first=1, n_recent=2)
        assert none is None and none_too is None and torch.equal(idx, got[0])
        assert torch.equal(md.view(torch.int32), got[3].view(torch.int32))


@pytest.mark.parametrize("N", [16384, 16657, 24581, 33280, 40964, 73730, 80001])
@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "odd"])
def test_long_caches(hippo, N, kind):
    for keep, first, recent in ((N // 2, 4, 256), (N // 10, 0, 1), (N - 1, 1, 0)):
        mass, k, v = make(1, 2, N, 64, "bf16", N, kind)
        check(hippo.hippo_evict_kv(mass, keep, k, v, n_first=first, n_recent=recent), mass, k, v, keep, first, recent, (N, keep))


def test_many_heads(hippo):
    for B, Hkv, N, keep in ((40, 8, 700, 300), (3, 97, 1500, 64), (4, 8, 9000, 4500)):
        mass, k, v = make(B, Hkv, N, 64, "bf16", B, "heavy")
        check(hippo.hippo_evict_kv(mass, keep, k, v, n_first=3, n_recent=9), mass, k, v, keep, 3, 9, (B, Hkv))


@pytest.mark.parametrize("kind", ["odd", "equal"])
def test_values_that_are_no_sums_and_equal_ones(hippo, kind):
    mass, k, v = make(2, 2, 3001, 64, "bf16", 9, kind)
    for keep, first, recent in ((1500, 4, 100), (2990, 0, 0), (300, 0, 0)):
        check(hippo.hippo_evict_kv(mass, keep, k, v, n_first=first, n_recent=recent), mass, k, v, keep, first, recent, kind)


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_strided_caches_fewer_rows_and_rows_behind(hippo, dtype):
    B, Hkv, N, d, keep = 2, 3, 500, 64, 200
    mass, k, v = make(B, Hkv, N, d, dtype, 1)
    # caches laid out [B, N, Hkv, d], a mass with a head stride of its own, 450 of the rows in use
    k2, v2 = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    wide = torch.full((B, Hkv + 1, N + 13), 1e9, device="cuda")
    wide[:, :Hkv, :N] = mass
    capacity = [torch.full((B, Hkv, 333, d), 3, dtype=TYPES[dtype], device="cuda") for _ in range(2)]
    kd, vd = capacity
    md = torch.full((B, Hkv, 400), -5.0, device="cuda")
    idx = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    got = hippo.hippo_evict_kv(wide[:, :Hkv], keep, k2, v2, n_rows=450, n_first=2, n_recent=30, idx_out=idx, k_dst=kd, v_dst=vd,
                               mass_dst=md)
    assert got[0].data_ptr() == idx.data_ptr() and got[1].data_ptr() == kd.data_ptr() and got[3].data_ptr() == md.data_ptr()
    check(got, mass[:, :, :450], k[:, :, :450], v[:, :, :450], keep, 2, 30)
    assert (kd[:, :, keep:] == 3).all() and (vd[:, :, keep:] == 3).all() and (md[:, :, keep:] == -5.0).all()
    # the indices and mass alone
    only = hippo.hippo_evict_kv(mass, keep, None, None, n_rows=450, n_first=2, n_recent=30)
    assert only[1] is None and only[2] is None and torch.equal(only[0], idx) and torch.equal(only[3], md[:, :, :keep])


def test_refusals_of_the_library_are_errors(hippo):
    mass, k, v = make(1, 2, 50, 64, "bf16", 1)
    for more in (dict(keep=20, n_first=15, n_recent=6), dict(keep=20, k_dst=k, v_dst=v)):
        with pytest.raises(hippo.HippoError):
            hippo.hippo_evict_kv(mass, more.pop("keep"), k, v, **more)


def test_heads_far_apart(hippo):
    # element offsets of the last head beyond 32 bits, in a cache view of few rows
    d, N, keep = 128, 40, 25
    stride_h = (1 << 31) // d * d + d
    base = [torch.zeros(stride_h + N * d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    views = [x.as_strided((1, 2, N, d), (0, stride_h, d, 1)) for x in base]
    g = torch.Generator(device="cuda").manual_seed(2)
    for x in views:
        x.copy_(torch.randint(0, 256, (1, 2, N, d), generator=g, device="cuda", dtype=torch.uint8))
    mass = torch.rand((1, 2, N), generator=g, device="cuda")
    check(hippo.hippo_evict_kv(mass, keep, *views, n_first=1, n_recent=4), mass, *(x.contiguous() for x in views), keep, 1, 4)


@pytest.mark.parametrize("B,Hkv,N,keep", [(1, 2, 900, 400), (1, 4, 16657, 8192), (2, 8, 20000, 3000)])
def test_streams_graphs_and_repeats(hippo, B, Hkv, N, keep):
    sets = [make(B, Hkv, N, 64, "bf16", s) for s in (1, 2)]
    want = [hippo.hippo_evict_kv(*(m, keep, k, v), n_first=4, n_recent=32) for m, k, v in sets]
    for got, (m, k, v) in zip(want, sets):
        check(got, m, k, v, keep, 4, 32)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [hippo.hippo_evict_kv(m, keep, k, v, n_first=4, n_recent=32, stream=s) for (m, k, v), s in zip(sets, side)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for a, b in zip(got, want) for p, q in zip(a, b))
    m, k, v = (x.clone() for x in sets[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hippo.hippo_evict_kv(m, keep, k, v, n_first=4, n_recent=32)
    for i in (1, 0, 1, 0):
        for dst, src in zip((m, k, v), sets[i]):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want[i]))
        again = hippo.hippo_evict_kv(sets[i][0], keep, sets[i][1], sets[i][2], n_first=4, n_recent=32)
        assert all(torch.equal(p, q) for p, q in zip(again, want[i]))
