"""GPU parity: the weights that hippo_*_attention_mass sums, against softmax in 64 bits.

With u = 2^-24, A = scale sum_c |q_c k_c| and dz = (d + 4) u max_n A, which bounds a row's logit errors (products and sums of d terms in
fp32), a weight w = exp(z - m) / l is off by at most
  w (2 dz + u (4 |z|_max + n + 64)):  its own logit's error and that of l's; the exponent's product, difference and exponential twice
  (log2 e times 2 u |z| each way is below 4); the n additions that a term of l goes through, tiles of its slice and then slices.
A row of mass adds the rows' weights to what was there: + u (rows + 2) |mass|.
"""
import math

import pytest
import torch

from parity_util import assert_close, host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def make(B, H, Hkv, d, ctx, q_len, dtype, seed, sharp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = sharp * torch.randn((B, q_len, H, d), generator=g, device="cuda")
    k, v = (torch.randn((B, Hkv, ctx + q_len, d), generator=g, device="cuda") for _ in range(2))
    mass = torch.exp(torch.randn((B, Hkv, ctx), generator=g, device="cuda"))
    return q.to(TYPES[dtype]), k.to(TYPES[dtype]), v.to(TYPES[dtype]), mass


def reference(q, k, v, ctx, mass, splits, scale=None):
    """out, mass, bound on mass, in 64 bits"""
    B, n_q, H, d = q.shape
    Hkv, N = k.shape[1], ctx + n_q
    G, scale = H // Hkv, scale or 1.0 / math.sqrt(d)
    if not splits:
        splits = min(max(1, 256 // (B * Hkv * -(-G * n_q // 64))), -(-N // 32))
    adds = -(-N // 16) // splits + 2 + 24 + splits // 16
    out = torch.empty((B, n_q, H, d), dtype=torch.float64, device="cuda")
    total = torch.zeros((B, Hkv, N), dtype=torch.float64, device="cuda")
    if mass is not None:
        total[:, :, :ctx] = mass[:, :, :ctx].double()
    bound = U * (G * n_q + 2) * total.abs()
    for b in range(B):
        for h in range(Hkv):
            kk, vv = k[b, h, :N].double(), v[b, h, :N].double()
            for i in range(n_q):
                rows = q[b, i, h * G:(h + 1) * G].double()
                seen = ctx + i + 1
                z = (rows @ kk[:seen].T.contiguous()) * scale
                w = torch.softmax(z, 1)
                out[b, i, h * G:(h + 1) * G] = w @ vv[:seen]
                dz = (d + 4) * U * scale * (rows.abs() @ kk[:seen].abs().T.contiguous()).amax(1, keepdim=True)
                rel = 2 * dz + U * (4 * z.abs().amax(1, keepdim=True) + adds + 64)
                total[b, h, :seen] += w.sum(0)
                bound[b, h, :seen] += (w * rel).sum(0) + U * (G * n_q + 2) * w.sum(0)
    return out, total, bound


def check(got, ref, dtype, what=""):
    out, total, bound = ref
    assert_close(host(got[0]), out.cpu().numpy(), dtype, str(what))
    err = (got[1][:, :, :total.shape[2]].double() - total).abs()
    assert bool(torch.isfinite(got[1][:, :, :total.shape[2]]).all()), what
    assert bool((err <= bound + 1e-37).all()), (what, float((err / (bound + 1e-37)).max()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,d,ctx,q_len", [
    (1, 1, 1, 64, 0, 1),            # nothing but the new row
    (1, 4, 2, 128, 0, 5),           # new rows alone, causal among themselves
    (2, 6, 3, 64, 1, 1), (1, 8, 2, 64, 14, 1), (1, 8, 2, 64, 15, 1), (1, 8, 2, 64, 16, 2), (1, 7, 1, 128, 30, 3),
    (1, 4, 2, 64, 832, 1), (2, 28, 4, 128, 77, 1), (1, 28, 4, 128, 255, 1), (1, 28, 4, 128, 256, 1), (1, 28, 4, 128, 1895, 1),
    (1, 14, 2, 64, 4097, 6), (3, 8, 8, 128, 500, 5), (1, 64, 8, 128, 2000, 2), (1, 64, 8, 128, 1000, 3),
    (1, 16, 1, 64, 700, 1), (1, 17, 1, 64, 700, 1), (1, 32, 1, 128, 900, 1), (1, 33, 1, 128, 900, 1), (1, 48, 1, 64, 300, 1),
    (1, 28, 4, 128, 3001, 13),      # 91 rows
    (1, 8, 1, 64, 701, 25),         # 200 rows
    (1, 128, 1, 64, 100, 9),        # 1152 rows
    (1, 4, 2, 64, 33000, 1), (1, 28, 4, 128, 16640, 6), (4, 16, 8, 128, 9000, 1), (40, 8, 8, 64, 300, 1),
])
def test_weights_and_outputs(hippo, dtype, B, H, Hkv, d, ctx, q_len):
    for sharp in (1.0, 4.0):        # 4: a few tokens have all the weight
        q, k, v, mass = make(B, H, Hkv, d, ctx, q_len, dtype, ctx + H, sharp)
        call = hippo.hippo_draft_attention_mass if q_len == 1 else hippo.hippo_verify_attention_mass
        plain = hippo.hippo_draft_attention if q_len == 1 else hippo.hippo_verify_attention
        got = call(q, k, v, mass, ctx, want_lse=True)
        check(got, reference(q, k, v, ctx, mass, 0), dtype, sharp)
        out, lse = plain(q, k, v, ctx, want_lse=True)
        # the same probabilities, rounded alike, and slices' outputs rounded to bf16 or not; another number of slices may round them
        # relative to another maximum, by 2^-9 each
        assert_close(host(got[0]), host(out), dtype)
        assert bool(((lse - got[2]).abs() <= 2 ** -8 + 1e-5 * lse.abs()).all())
        # every row gives a weight of 1 in all
        fresh = call(q, k, v, None, ctx)[1]
        check((got[0], fresh), reference(q, k, v, ctx, None, 0), dtype, sharp)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,Hkv,d,ctx,q_len", [(4, 2, 64, 832, 1), (28, 4, 128, 1000, 6), (8, 1, 64, 301, 12)])
@pytest.mark.parametrize("splits", [1, 2, 7, 64, 5000])
def test_slices(hippo, dtype, H, Hkv, d, ctx, q_len, splits):
    q, k, v, mass = make(2, H, Hkv, d, ctx, q_len, dtype, splits, 2.0)
    got = hippo.hippo_verify_attention_mass(q, k, v, mass, ctx, num_splits=splits)
    check(got, reference(q, k, v, ctx, mass, min(splits, -(-(ctx + q_len) // 32))), dtype, splits)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,d,ctx,q_len", [
    (1, 16, 1, 64, 735, 1), (2, 6, 3, 128, 735, 1), (1, 16, 2, 128, 600, 2), (2, 5, 1, 64, 253, 3), (3, 4, 4, 128, 256, 16),
    (70, 8, 4, 64, 31, 2)])
def test_one_slice_in_one_launch(hippo, dtype, B, H, Hkv, d, ctx, q_len):
    """up to 16 rows over the whole cache in a block each, which sums the weights itself; in place, with appended rows"""
    q, k, v, mass = make(B, H, Hkv, d, ctx, q_len, dtype, 21, 2.0)
    got = hippo.hippo_verify_attention_mass(q, k, v, mass, ctx, want_lse=True, num_splits=1)
    check(got, reference(q, k, v, ctx, mass, 1), dtype)
    plain = hippo.hippo_verify_attention(q, k, v, ctx, want_lse=True, num_splits=1)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[2], plain[1])
    k_new, v_new = (x[:, :, ctx:].transpose(1, 2).contiguous() for x in (k, v))
    k2, v2 = k.clone(), v.clone()
    k2[:, :, ctx:], v2[:, :, ctx:] = 3.0, float("nan")
    room = torch.full((B, Hkv, ctx + q_len + 5), 50.0, device="cuda")
    room[:, :, :ctx] = mass
    again = hippo.hippo_verify_attention_mass(q, k2, v2, room, ctx, mass_out=room, k_new=k_new, v_new=v_new, num_splits=1)
    assert torch.equal(again[0], got[0]) and torch.equal(room[:, :, :ctx + q_len], got[1])
    assert (room[:, :, ctx + q_len:] == 50.0).all() and torch.equal(k2, k) and torch.equal(v2, v)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,d,ctx,q_len", [
    (1, 4, 2, 64, 832, 1), (2, 28, 4, 128, 500, 6), (1, 28, 4, 128, 1895, 1), (3, 8, 4, 64, 40, 3), (1, 28, 4, 128, 16640, 6),
    (1, 8, 1, 128, 700, 25)])
def test_appended_rows(hippo, dtype, B, H, Hkv, d, ctx, q_len):
    q, k, v, mass = make(B, H, Hkv, d, ctx, q_len, dtype, 3, 2.0)
    want = hippo.hippo_verify_attention_mass(q, k, v, mass, ctx)
    k2, v2 = k.clone(), v.clone()
    k2[:, :, ctx:], v2[:, :, ctx:] = 77.0, float("nan")            # what rejected rows left there
    stale = torch.full((B, Hkv, ctx + q_len + 9), 50.0, device="cuda")
    stale[:, :, :ctx] = mass
    k_new, v_new = (x[:, :, ctx:].transpose(1, 2).contiguous() for x in (k, v))
    got = hippo.hippo_verify_attention_mass(q, k2, v2, stale, ctx, mass_out=stale, k_new=k_new, v_new=v_new)
    assert got[1].data_ptr() == stale.data_ptr()
    assert torch.equal(got[0], want[0]) and torch.equal(stale[:, :, :ctx + q_len], want[1])
    assert (stale[:, :, ctx + q_len:] == 50.0).all()
    assert torch.equal(k2, k) and torch.equal(v2, v)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strides_scale_and_given_buffers(hippo, dtype):
    B, H, Hkv, d, ctx, q_len = 2, 14, 2, 64, 333, 2
    q, k, v, mass = make(B, H, Hkv, d, ctx, q_len, dtype, 8)
    ref = reference(q, k, v, ctx, mass, 0, 0.31)
    wide = [torch.full((B, ctx + 100, Hkv, 2 * d), 1e4, dtype=k.dtype, device="cuda") for _ in range(2)]
    views = [w[..., :d].transpose(1, 2) for w in wide]
    for view, x in zip(views, (k, v)):
        view[:, :, :ctx + q_len] = x
    m_in = torch.full((Hkv, B, ctx + 31), 9.0, device="cuda").transpose(0, 1)
    m_in[:, :, :ctx] = mass
    m_out = torch.full((B, Hkv + 2, ctx + q_len + 5), -3.0, device="cuda")[:, 1:Hkv + 1]
    out = torch.empty_like(q)
    ws = torch.empty(hippo.load().hippo_attention_mass_workspace_bytes(hippo.kv_desc(views[0], H), q_len, ctx + q_len, 0),
                     dtype=torch.uint8, device="cuda")
    got = hippo.hippo_verify_attention_mass(q, *views, m_in, ctx, softmax_scale=0.31, out=out, mass_out=m_out, workspace=ws)
    check(got, ref, dtype)
    assert got[0].data_ptr() == out.data_ptr() and got[1].data_ptr() == m_out.data_ptr()
    assert (m_out[:, :, ctx + q_len:] == -3.0).all() and (m_in[:, :, ctx:] == 9.0).all()
    with pytest.raises(hippo.HippoError):
        hippo.hippo_verify_attention_mass(q, *views, m_in, ctx, workspace=ws[:-256])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,d,ctx,q_len,splits", [
    (8, 64, 200, 1, 0), (8, 128, 200, 3, 1), (8, 128, 1895, 1, 0), (28, 64, 900, 6, 7), (64, 128, 3001, 4, 0), (8, 64, 4097, 1, 64)])
def test_infinite_and_nan_logits(hippo, dtype, H, d, ctx, q_len, splits):
    """as a softmax has them, each in its KV head: logits of -inf give no weight (what lies at their rows is added to nothing),
    one of +inf or NaN makes the head's weights and outputs NaN, and so do rows of -inf alone"""
    q, k, v, mass = make(2, H, 4, d, ctx, q_len, dtype, 17)
    q[..., 0] = q[..., 0].abs() + 0.5                            # so that a channel of -inf gives a logit of -inf
    call = lambda k: hippo.hippo_verify_attention_mass(q, k, v, mass, ctx, want_lse=True, num_splits=splits)
    clean, odd = call(k), k.clone()
    gone = torch.zeros(ctx + q_len, dtype=torch.bool, device="cuda")
    gone[:70], gone[ctx - 3:ctx] = True, True                     # whole tiles, and a piece of the last
    odd[0, 1, gone, 0] = -math.inf
    odd[0, 2, 5, 3] = math.nan
    odd[0, 3, ctx // 2, 0] = math.inf
    odd[1, 0, :, 0] = -math.inf
    odd[1, 2, 0, 0] = -math.inf
    out, total, lse = call(odd)
    of_head = lambda x, b, h: x[b, :, h * (H // 4):(h + 1) * (H // 4)]
    for b, h in ((0, 2), (0, 3), (1, 0)):
        assert bool(of_head(out, b, h).isnan().all()) and bool(total[b, h].isnan().all())
    for b, h in ((0, 0), (1, 1), (1, 3)):                         # the heads beside them
        assert torch.equal(of_head(out, b, h), of_head(clean[0], b, h)) and torch.equal(total[b, h], clean[1][b, h])
        assert torch.equal(lse[b, h * (H // 4):(h + 1) * (H // 4)], clean[2][b, h * (H // 4):(h + 1) * (H // 4)])
    assert torch.equal(total[0, 1, gone], mass[0, 1, gone[:ctx]]) and torch.equal(total[1, 2, :1], mass[1, 2, :1])
    # the others' weights are those of a cache without these rows, whose terms go through up to as many additions more
    for b, h, rows in ((0, 1, gone), (1, 2, torch.arange(ctx + q_len, device="cuda") == 0)):
        left, n = ~rows, int(rows.sum())
        ref = reference(of_head(q, b, h)[None].contiguous(), k[b:b + 1, h:h + 1, left].contiguous(), v[b:b + 1, h:h + 1, left].contiguous(),
                        ctx - n, mass[b:b + 1, h:h + 1, left[:ctx]].contiguous(), splits)
        more = U * n * (ref[1] - torch.nn.functional.pad(mass[b:b + 1, h:h + 1, left[:ctx]].double(), (0, q_len))).abs()
        check((of_head(out, b, h)[None], total[b:b + 1, h:h + 1, left]), (ref[0], ref[1], ref[2] + more), dtype, (b, h))


def test_heads_far_apart(hippo):
    # the second KV head lies more than 2^32 bytes, and 2^31 elements, behind the first
    H, d, ctx = 4, 64, 200
    q, k, v, mass = make(1, H, 2, d, ctx, 1, "bf16", 4)
    stride = (1 << 31) + d
    far = [torch.empty(stride + (ctx + 1) * d, dtype=torch.bfloat16, device="cuda").as_strided((1, 2, ctx + 1, d), (0, stride, d, 1))
           for _ in range(2)]
    for f, x in zip(far, (k, v)):
        f.copy_(x)
    want = hippo.hippo_draft_attention_mass(q, k, v, mass, ctx)
    got = hippo.hippo_draft_attention_mass(q, *far, mass, ctx)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,Hkv,d,ctx,q_len", [(4, 2, 64, 832, 1), (28, 4, 128, 5000, 6)])
def test_streams_graphs_and_repeats(hippo, dtype, H, Hkv, d, ctx, q_len):
    sets = [make(1, H, Hkv, d, ctx, q_len, dtype, s) for s in (1, 2)]
    want = [hippo.hippo_verify_attention_mass(q, k, v, m, ctx) for q, k, v, m in sets]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [hippo.hippo_verify_attention_mass(q, k, v, m, ctx, stream=s) for (q, k, v, m), s in zip(sets, side)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for a, b in zip(got, want) for p, r in zip(a, b))
    q, k, v, m = (x.clone() for x in sets[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hippo.hippo_verify_attention_mass(q, k, v, m, ctx)
    for i in (1, 0, 1, 0):
        for dst, src in zip((q, k, v, m), sets[i]):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, r) for p, r in zip(held, want[i]))
        again = hippo.hippo_verify_attention_mass(*sets[i], ctx)
        assert all(torch.equal(p, r) for p, r in zip(again, want[i]))
