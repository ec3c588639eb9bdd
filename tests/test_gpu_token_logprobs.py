"""GPU parity: hippo_token_logprobs against log-softmax, entropy and ranking in 64 bits.

Words and their order are whole numbers on identical inputs: equal.  Values are fp32 sums of n words (at most ceil(V / 256) in a
row on one lane, plus the joins), so with u = 2^-24, t = (x - M) / T, p = softmax, rest = the share of the words below the maximum:
  |log Z  error| <= u ((n + 64) rest + 4 log Z)        a weight's own error, 2 |t| u and the exponential's, is within the 64
                                                       (rest has no word with |t| > 104, whose weight is 0)
  |log p  error| <= that + 4 u |t|
  |H      error| <= u ((n + 64) (rest + sum p |t|) + 4 sum p t^2 + 4 H)
The sum of p t^2 stands for t's own two roundings inside t exp(t).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def reference(x, tokens, T, n_top):
    """per row: log p of the token, entropy, ids, log p of them, and the bounds"""
    x = x.astype(np.float64)
    R, V = x.shape
    n = -(-V // 256)
    out = []
    for r in range(R):
        m = x[r].max()
        ids = np.lexsort((np.arange(V), -x[r]))[:n_top]
        if m == -np.inf:
            out.append((-np.inf, 0.0, ids, np.full(n_top, -np.inf), 0.0, 0.0, np.zeros(n_top)))
            continue
        t = (x[r] - m) / T
        e = np.exp(t)
        Z = e.sum()
        # log Z = log1p(Z - 1), whose rest keeps its bits where the best word has nearly all the weight
        rest = e[x[r] < m].sum()
        log_z = math.log1p((x[r] == m).sum() - 1 + rest)
        p = e / Z
        live = e > 0
        h1 = -(p[live] * t[live]).sum()
        H = log_z + h1
        bz = U * ((n + 64) * rest / Z + 4 * log_z)
        lp = t - log_z
        tok = int(tokens[r])
        with np.errstate(invalid="ignore"):
            at = lambda w: bz + 4 * U * np.where(np.isinf(t[w]), 0.0, np.abs(t[w]))
        lt, bt = (lp[tok], float(at(tok))) if 0 <= tok < V else (-np.inf, 0.0)
        bh = U * ((n + 64) * (rest / Z + h1) + 4 * (p[live] * t[live] ** 2).sum() + 4 * H)
        out.append((lt, H, ids, lp[ids], bt, bh, at(ids)))
    return [np.array(c) for c in zip(*out)]


def check(got, ref, what=""):
    lt, H, ids, lp, bt, bh, bl = ref
    got = [g.cpu().numpy().reshape(len(lt), -1) for g in got]

    def near(g, want, bound, name):
        g, want, bound = g.reshape(want.shape).astype(np.float64), want, bound + 1e-37
        fine = np.isfinite(want)
        assert np.array_equal(g[~fine], want[~fine]), (what, name)
        err = np.abs(g[fine] - want[fine])
        assert np.all(err <= bound[fine]), (what, name, float((err / bound[fine]).max()))
    near(got[0], lt, bt, "logprob")
    near(got[1], H, bh, "entropy")
    if ids.shape[1]:
        np.testing.assert_array_equal(got[2], ids, err_msg=str(what))
        near(got[3], lp, bl, "top_logprobs")


def padded(x, dtype):
    """the rows on the GPU, garbage behind the vocabulary"""
    R, V = x.shape
    full = torch.full((R, -(-V // 8) * 8 + 8), 999.0, dtype=TYPES[dtype], device="cuda")
    full[:, :V] = torch.from_numpy(x.astype(np.float32)).cuda()
    return full[:, :V]


def run(hippo, x, tokens, dtype, T=1.0, n_top=5, what=""):
    d = padded(x, dtype)
    seen = d.float().cpu().numpy()
    tok = torch.from_numpy(np.asarray(tokens, np.int32)).cuda()
    got = hippo.hippo_token_logprobs(d, tok, T, n_top=n_top)
    assert len(got) == (4 if n_top else 2)
    torch.cuda.synchronize()
    check(got, reference(seen, tokens, T, n_top), what)
    return got


def lm_rows(r, R, V, masked=0.01):
    x = 2.0 * r.standard_normal((R, V))
    for row in x:
        row[r.integers(0, V, 3)] = row.max() + r.uniform(0, 4, 3)
    x[r.random((R, V)) < masked] = -np.inf
    return x


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,V,n_top", [
    (1, 1, 1), (3, 2, 2), (2, 7, 7), (4, 63, 0), (3, 64, 32), (2, 255, 5), (2, 257, 20), (2, 1000, 31),
    (1, 8192, 5), (5, 8193, 1), (1, 32000, 5), (2, 32768, 32), (3, 32769, 32), (6, 152064, 20), (1, 1 << 20, 32),
    (256, 3000, 4), (257, 3000, 4), (300, 33001, 3), (1025, 9001, 2), (1030, 40000, 20),
])
def test_sizes(hippo, dtype, R, V, n_top):
    r = np.random.default_rng(R * 7 + V)
    run(hippo, lm_rows(r, R, V), r.integers(0, V, R), dtype, n_top=n_top)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,V", [(2, 5000), (3, 40000), (1100, 20000)])
def test_equal_logits_come_in_word_order(hippo, dtype, R, V):
    r = np.random.default_rng(V)
    for x in (np.zeros((R, V)), r.integers(-2, 3, (R, V)).astype(float), np.where(r.random((R, V)) < 0.5, 0.0, -0.0)):
        run(hippo, x, r.integers(0, V, R), dtype, n_top=32)
    x = np.full((R, V), -1.0)                                     # few above many equal
    x[:, V - 3:] = 1.0
    x[:, V // 2] = 0.5
    run(hippo, x, r.integers(0, V, R), dtype, n_top=7)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,V", [(2, 3000), (2, 40000), (1100, 20000)])
def test_rows_in_order(hippo, dtype, R, V):
    # every word larger than all before it (each is a candidate when it is met), and the other way round
    up = np.tile(np.linspace(-8.0, 8.0, V), (R, 1))
    for x in (up, up[:, ::-1]):
        run(hippo, x, np.arange(R) % V, dtype, n_top=20)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masked_words_and_words_outside(hippo, dtype):
    V, r = 20001, np.random.default_rng(3)
    x = lm_rows(r, 8, V)
    x[0] = -np.inf                                                # nothing left
    x[1] = -np.inf
    x[1, 17] = -3.0                                               # one word left
    x[2, :V - 4] = -np.inf                                        # fewer words than asked for
    x[3, ::2] = -np.inf
    tokens = np.array([5, 17, 0, 2, -1, V, 1 << 30, 4])
    got = run(hippo, x, tokens, dtype, n_top=10)
    assert got[0][1] == 0 and got[1][1] == 0 and got[1][0] == 0   # certain: log p 0, entropy 0
    assert torch.isinf(got[0][[0, 2, 3, 4, 5, 6]]).all()
    x = np.full((1100, 700), -np.inf)                             # the route of many rows
    x[1::2, 3] = 1.0
    run(hippo, x, np.full(1100, 3), dtype, n_top=4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_nan_stays_in_its_row_and_words_in_the_vocabulary(hippo, dtype):
    for R, V in ((3, 500), (3, 40000), (1100, 500)):
        r = np.random.default_rng(R + V)
        x = lm_rows(r, R, V)
        x[1, 7] = np.nan
        got = hippo.hippo_token_logprobs(padded(x, dtype), torch.zeros(R, dtype=torch.int32, device="cuda"), n_top=32)
        others = np.arange(R) != 1
        seen = padded(x, dtype).float().cpu().numpy()
        check([g[torch.from_numpy(others).cuda()] for g in got], reference(seen[others], np.zeros(R - 1, int), 1.0, 32))
        assert torch.isnan(got[0][1]) and torch.isnan(got[1][1]) and torch.isnan(got[3][1]).all()
        assert ((got[2] >= 0) & (got[2] < V)).all()
    for fill in (np.nan, np.inf):
        got = hippo.hippo_token_logprobs(padded(np.full((2, 40000), fill), dtype), torch.zeros(2, dtype=torch.int32, device="cuda"),
                                         n_top=32)
        assert ((got[2] >= 0) & (got[2] < 40000)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [0.05, 0.7, 30.0])
def test_temperatures_and_rows_with_one_likely_word(hippo, dtype, T):
    r = np.random.default_rng(11)
    for R, V in ((4, 32000), (2, 152064)):
        x = lm_rows(r, R, V)
        x[0] += 4000.0                                            # far from 0
        x[1, 100] = x[1].max() + 9.0                              # the others weigh little
        x[1, 200] = x[1, 100]
        run(hippo, x, r.integers(0, V, R), dtype, T=T, n_top=8)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_nearly_certain_word_keeps_its_entropy(hippo, dtype):
    # 1 + rest in 32 bits would leave one digit of the rest, 1e-6 here, or none
    V = 30000
    x = np.full((3, V), -26.0)
    x[:, 4321] = 0.0
    x[1, 5] = -15.0
    x[2] -= 20.0
    x[2, 4321] = 0.0
    got = run(hippo, x, np.full(3, 4321), dtype, n_top=3)
    assert (got[0][:2] < 0).all() and (got[1][:2] > 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_leading_dimensions_strides_and_given_buffers(hippo, dtype):
    r = np.random.default_rng(5)
    B, n, V = 3, 4, 5001
    x = torch.from_numpy(lm_rows(r, B * n, V).reshape(B, n, V)).to(TYPES[dtype]).cuda()
    wide = torch.full((B, n, 5016), 50.0, dtype=x.dtype, device="cuda")
    wide[..., :V] = x
    tokens = torch.from_numpy(r.integers(0, V, (B, n)).astype(np.int32)).cuda()
    flat = hippo.hippo_token_logprobs(wide.view(B * n, 5016)[:, :V], tokens.view(-1), 0.9, n_top=3)
    given = [torch.empty((B, n), device="cuda"), torch.empty((B, n), device="cuda"),
             torch.empty((B, n, 3), dtype=torch.int32, device="cuda"), torch.empty((B, n, 3), device="cuda")]
    got = hippo.hippo_token_logprobs(wide[..., :V], tokens, 0.9, 3, *given)
    for a, b, c in zip(got, flat, given):
        assert a.data_ptr() == c.data_ptr() and torch.equal(a.reshape(b.shape), b)
    check(flat, reference(x.view(B * n, V).float().cpu().numpy(), tokens.view(-1).cpu().numpy(), 0.9, 3))
    last = hippo.hippo_token_logprobs(wide[:, -1, :V], tokens[:, -1].contiguous(), 0.9, n_top=3)   # rows n apart
    for a, b in zip(last, got):
        assert torch.equal(a, b[:, -1])
    one = hippo.hippo_token_logprobs(x[1, 2:3].clone(), tokens[1, 2:3].contiguous(), 0.9, n_top=3)   # one row needs no spacing
    for a, b in zip(one, got):
        assert torch.equal(a[0], b[1, 2])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_stride_of_the_only_row_is_nobodys(hippo, dtype):
    g = torch.Generator(device="cuda").manual_seed(12)
    tokens = torch.tensor([4999], dtype=torch.int32, device="cuda")
    wide = (2.0 * torch.randn((3, 6001), generator=g, device="cuda")).to(TYPES[dtype])       # rows of no multiple of 16 bytes
    chain = (2.0 * torch.randn((1, 7, 32004), generator=g, device="cuda")).to(TYPES[dtype])
    for x in (wide[0:1, :5000], wide[0:1], chain[:, -1], chain[:, -1:], chain[0, -1:, :5000]):
        t = tokens.view(x.shape[:-1])
        got = hippo.hippo_token_logprobs(x, t, 0.8, n_top=5)
        check(got, reference(x.reshape(1, -1).float().cpu().numpy(), [4999], 0.8, 5), x.shape)


@pytest.mark.parametrize("R,V", [(2, 152064), (1100, 9000), (4, 30000)])
def test_streams_graphs_and_repeats(hippo, R, V):
    g = torch.Generator(device="cuda").manual_seed(R)
    sets = [(3 * torch.randn((R, V), generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2)]
    tok = torch.randint(0, V, (R,), generator=g, device="cuda", dtype=torch.int32)
    want = [hippo.hippo_token_logprobs(x, tok, n_top=20) for x in sets]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):                                            # two calls at once, each on its own stream
        got = [hippo.hippo_token_logprobs(x, tok, n_top=20, stream=s) for x, s in zip(sets, side)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    x = sets[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = hippo.hippo_token_logprobs(x, tok, n_top=20)
    for k in (1, 0, 1, 0):
        x.copy_(sets[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want[k]))
        again = hippo.hippo_token_logprobs(sets[k], tok, n_top=20)
        assert all(torch.equal(p, q) for p, q in zip(again, want[k]))
