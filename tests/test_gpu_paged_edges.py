"""Inputs of the paged-cache calls where an answer hangs on one step of a kernel, against the 64-bit oracle."""
import itertools

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2511_12201_amd import binding as ob
from test_gpu_paged import BF16, F32, U32, Cache, Guarded, attend_bars, check_attention, check_eviction, host, ints, rand, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("D,rows,n", [(128, 250000, 40), (64, 250000, 40), (128, 9000, 40), (64, 3000, 300), (128, 5000, 9), (128, 90000, 2)])
def test_what_one_row_dominates_is_its_v(D, rows, n):
    """Every query row's score on one cache row of its own is 21 to 25, on the others 0: these weigh 250000 exp(-21) < 2e-4 together,
    so O is that row's V to one rounding, whatever the fraction of the score.  The rows are anywhere among the tiles."""
    rng = np.random.default_rng(rows + D)
    H, marks, page_rows = 4, 32, 256
    cache = Cache(rng, 1, 1, -(-rows // page_rows), page_rows, D, BF16)
    cache.K.zero_()
    V = cache.V[cache.table[0, 0].long()].reshape(-1, D)
    where = np.sort(rng.choice(rows - n, marks, replace=False))
    for m, j in enumerate(where):
        cache.K[cache.table[0, 0, j // page_rows].long(), j % page_rows, m] = 1.0
    mark = rng.integers(0, marks, (H, n))
    score = rng.uniform(21, 25, (H, n))
    Q = torch.zeros(1, H, n, D, dtype=BF16, device="cuda")
    for i, t in itertools.product(range(H), range(n)):
        Q[0, i, t, mark[i, t]] = float(score[i, t])
    desc = ob.make_chunk_desc(Q, n_kv_heads=1, softmax_scale=1.0)
    acc = torch.zeros(1, 1, cache.cap, device="cuda")
    O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints([[rows]]), ints([n]), acc_out=acc)
    z = host(Q.amax(-1))[0]                                  # the scores, exactly
    seen = rows - n + 1 + np.arange(n)[None]
    rest = (seen - 1) * np.exp(-z)                            # the others' weights, as shares of the row's
    v = host(V)[where][mark]                                  # [H, n, D]
    # the others move O by rest (|v| + 5), their sums are exact to 2^-8; V itself is a bf16 number and may not move a whole step
    want = v / (1 + rest)[..., None]
    within(host(O)[0], want, 2.0 ** -9 * np.abs(v) * 1.01 + 2 * rest[..., None] * (np.abs(v) + 6), "O")
    # score and sum in fp32; 2^x and log2 are off by a few steps.  The sum is 1 and many numbers too small to move it by more than a
    # step: an addition rounds by up to half a step of 1, 2^-24, for each of the up to 256 spans that share the rows and are joined one
    # after the other, and for each of the up to 16 tiles of the span, in both halves of a wavefront.
    within(host(lse)[0], z + np.log1p(rest), 6 * U32 * 25 + 2.0 ** -20 + (256 + 2 * 16) * U32, "lse")
    p = 1 / (1 + rest)
    got = host(acc)[0, 0, where]
    for m, j in enumerate(where):
        # a weight is off by the roundings of its exponent, 25 log2 e at most, and of the log-sum-exp
        count = (mark == m).sum()
        assert abs(got[m] - p[mark == m].sum() - rest_weight(z, seen, mark == m)) <= count * 12 * U32 * 37 + 1e-4


def rest_weight(z, seen, own):
    """What the query rows of the other marks leave on a row: exp(-z) of each, a few 1e-10."""
    return np.exp(-z[~own]).sum()


def exact_scores(rng, cache, Q):
    """Q and K of -1, 0 and 1: a score is a whole number, whatever order its sum is taken in."""
    cache.K.copy_(torch.from_numpy(rng.integers(-1, 2, cache.K.shape).astype(np.float32)))
    Q.copy_(torch.from_numpy(rng.integers(-1, 2, Q.shape).astype(np.float32)))


@pytest.mark.parametrize("H,n,rows", [(7, 1, 60), (7, 4, 200), (32, 1, 300), (1, 32, 90), (3, 2, 17)])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_few_query_rows_keep_17_bits(H, n, rows, D):
    rng = np.random.default_rng(rows)
    cache = Cache(rng, 1, 1, -(-rows // 16), 16, D, BF16)
    Q = torch.zeros(1, H, n, D, dtype=BF16, device="cuda")
    exact_scores(rng, cache, Q)
    desc = ob.make_chunk_desc(Q, n_kv_heads=1, softmax_scale=0.25)
    O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints([[rows]]), ints([n]))
    wO, wl, _, pv, qk = po.attend(host(Q), cache.oracle(), np.array([[rows]]), [n], True, 0.25)
    # exponents below 32 log2 e with two roundings, 2^x off by 2^-22, `rows` additions in numerator and sum; a weight as two
    # numbers of 8 bits is off by 2^-17; half a step of the output
    e = 2 * (2 * 47 * U32 + 2.0 ** -22) + 2 * rows * U32 + 2.0 ** -17
    within(host(O), wO, e * pv + 2.0 ** -8 * np.abs(wO), "O")
    within(host(lse), wl, 2 * (2 * 47 * U32 + 2.0 ** -22) + rows * U32 + 4 * U32 * np.abs(wl), "lse")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 30, 200])
def test_an_fp32_score_is_a_sum_of_short_sums(D, n):
    """A product of 1 and D - 1 of just over a quarter of a step of 1: added to the 1 one by one they are lost, by pairs each rounds up, so
    that one chain is off by about D / 4 steps of 1.  One row is seen: its log-sum-exp is the score, its weight 1 a query row."""
    rng = np.random.default_rng(0)
    small = 0.51 * 2.0 ** -24
    cache = Cache(rng, 1, 1, 1, 16, D, F32)
    cache.K.fill_(2.0 ** -12)
    Q = torch.full((1, 2, n, D), small * 2.0 ** 12, device="cuda")
    Q[..., 0], cache.K[..., 0] = 1.0, 1.0
    desc = ob.make_chunk_desc(Q, n_kv_heads=1, causal=False, softmax_scale=1.0)
    acc = torch.zeros(1, 1, 16, device="cuda")
    O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints([[1]]), ints([n]), acc_out=acc)
    # 31 small products are added to the 1, each off by no more than itself (one by one: lost) or by half a step for each pair; three
    # additions of the sums round by half a step; the exponent's and the logarithm's scale are two products with rounded constants
    bar = (31 * 0.51 + 3 + 5) * 2.0 ** -24
    within(host(lse), 1 + (D - 1) * small, bar, "lse")
    # the same scores in the weights: what is left is the rounding of their logarithms' scale, and 2 n ones are added
    assert abs(float(acc[0, 0, 0]) - 2 * n) <= 2 * n * (8 + 2 * n) * 2.0 ** -24
    assert torch.equal(O, cache.V[cache.table[0, 0, 0].long(), 0].expand_as(O))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,end", [(3, 70), (10, 430), (40, 430), (300, 430), (600, 900)])
def test_a_nan_token_leaves_the_rows_it_does_not_see_alone(dtype, n, end):
    """One query row of one token is NaN: the weights of the rows that it sees are, those behind them and on a page that is missing are
    what they were without it."""
    rng = np.random.default_rng(n)
    cache = Cache(rng, 1, 1, -(-end // 16), 16, 64, dtype)
    cache.table[0, 0, 1] = -1
    Q = rand(rng, 1, 3, n, 64, dtype=dtype)
    desc, token = ob.make_chunk_desc(Q, n_kv_heads=1), n // 2
    out = []
    for value in (None, float("nan")):
        if value is not None:
            Q[0, 1, token, 7] = value
        acc = torch.full((1, 1, cache.cap), 0.5, device="cuda")
        out.append((*ob.omni_paged_attn(desc, Q, cache.pool, ints([[end]]), ints([n]), acc_in=acc, acc_out=acc), acc[0, 0]))
    (O, lse, acc), (bad_O, bad_lse, bad) = out
    seen = end - n + token + 1
    there = torch.arange(cache.cap, device="cuda") // 16 != 1
    assert bad[:seen][there[:seen]].isnan().all() and (bad[:end][~there[:end]] == 0.5).all() and (bad[end:] == 0.5).all()
    assert torch.equal(bad[seen:], acc[seen:])               # the other tokens' weights, in the same order
    assert bad_O[0, 1, token].isnan().all() and bad_lse[0, 1, token].isnan()
    clean = torch.ones(3, n, dtype=torch.bool, device="cuda")
    clean[1, token] = False
    assert torch.equal(bad_O[0][clean], O[0][clean]) and torch.equal(bad_lse[0][clean], lse[0][clean])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [6, 40])
def test_attention_after_an_append_that_ran_over(dtype, n):
    """Sequence 0 has room for 4 of its tokens: with the counts of what was stored these see what they should and the others nothing;
    sequence 1, which fits, is not affected."""
    rng = np.random.default_rng(n)
    cache = Cache(rng, 2, 2, 8, 16, 64, dtype)
    Q, K, V = (rand(rng, 2, h, n, 64, dtype=dtype) for h in (4, 2, 2))
    cap, pos = cache.cap, torch.zeros(2, 2, cache.cap, dtype=torch.int32, device="cuda")
    have = [cap - 4, 20]
    _, end = ob.omni_paged_append(ob.make_chunk_desc(Q, K), None, None, K, V, cache.pool, ints(have), ints([n, n]),
                                  ints([[h, h] for h in have]), pos)
    assert end.tolist() == [[cap, cap], [20 + n, 20 + n]]
    stored = [min(n, cap - h) for h in have]
    O, lse, _ = check_attention(cache, Q, end.tolist(), stored, True, True, dtype)
    assert not O[0, :, 4:].any() and torch.isneginf(lse[0, :, 4:]).all()
    # the oracle on sequence 0 with the rows that it had and each stored token's own behind them, one token at a time
    pool = cache.oracle()
    for t in range(4):
        wO, _, _, pv, qk = po.attend(host(Q[:1, :, t:t + 1]), pool, np.full((1, 2), have[0] + t + 1), [1], False, 0.125)
        bar = (2 * ((64 + 2) * U32 * qk + 2.0 ** -21) + 2 * cap * U32)[..., None] * pv + (2 * 2.0 ** -8 * pv + 2.0 ** -8 * np.abs(wO)) * (dtype is BF16) + U32
        within(host(O[:1, :, t:t + 1]), wO, bar, f"token {t}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("G,n,end,page_rows,D", [
    (1, 1, 700, 16, 64), (7, 1, 9001, 64, 128), (4, 8, 5003, 32, 64), (4, 9, 4000, 16, 128), (7, 40, 33001, 16, 128), (2, 130, 8321, 256, 64),
    (1, 300, 300, 64, 128), (3, 257, 2050, 16, 64), (8, 64, 66000, 16, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_every_row_counts_once(G, n, end, page_rows, D, causal, dtype):
    """All scores are 0: every weight is 1, sums are whole numbers, the log-sum-exp is the logarithm of the number of rows seen.  Column
    c of V marks up to 32 rows of the cache, the first and last of its tiles and windows before others: O times the number of
    rows is how many of them a token sees, and 1 / 32 of that is far above a bf16 rounding."""
    rng = np.random.default_rng(end)
    Hkv, B = 2, 1
    cache = Cache(rng, B, Hkv, -(-end // page_rows), page_rows, D, dtype)
    cache.K.zero_()
    cache.V.zero_()
    ends = [end, end - 13]
    j = np.arange(end)
    border = np.flatnonzero((j % 64 < 2) | (j % 64 > 61) | (j % 32 == 0) | (j % 32 == 31))
    first = np.concatenate([rng.permutation(border), rng.permutation(np.setdiff1d(j, border))])[:32 * D]
    column = np.full(end, -1)
    column[first] = np.arange(len(first)) % D
    table = cache.table.cpu().numpy()
    for g in range(Hkv):
        at = torch.from_numpy(table[0, g, first // page_rows].astype(np.int64)).cuda()
        cache.V[at, torch.from_numpy(first % page_rows).cuda(), torch.from_numpy(column[first]).cuda()] = 1.0
    cache.poison([ends])
    Q = rand(rng, B, Hkv * G, n, D, dtype=dtype)
    acc = torch.zeros(B, Hkv, cache.cap, device="cuda")
    O, lse = ob.omni_paged_attn(ob.make_chunk_desc(Q, n_kv_heads=Hkv, causal=causal), Q, cache.pool, ints([ends]), ints([n]), acc_out=acc)
    for g, e in enumerate(ends):
        seen = np.maximum(e - n + 1 + np.arange(n), 0) if causal else np.full(n, e)
        marks = np.zeros((end + 1, D))
        marks[1:][first, column[first]] = 1
        count = marks.cumsum(0)[seen]                                # [n, D] marked rows that a token sees
        heads = slice(g * G, (g + 1) * G)
        want = count / np.maximum(seen, 1)[:, None]
        # 1 / sum, the product with it, the store
        within(host(O)[0, heads], np.broadcast_to(want, (G, n, D)), want * ((2.0 ** -8 if dtype is BF16 else U32) + 3 * U32), "O")
        with np.errstate(divide="ignore"):
            log = np.log(seen.astype(np.float64))
        # log2 off by four steps of its size, times a rounded constant
        within(host(lse)[0, heads], np.broadcast_to(log, (G, n)), 6 * 2 * U32 * np.abs(np.where(seen > 0, log, 0)), "lse")
        share = np.where(seen > 0, G / np.maximum(seen, 1), 0.0)
        w = np.zeros(e)
        for t in range(n):
            w[:seen[t]] += share[t]
        # an exponent below 17 with three roundings, 2^x off by 2^-22, G n additions
        within(host(acc)[0, g, :e], w, (3 * 2 * 17 * U32 + 2.0 ** -21 + G * n * U32) * w, "weights")


TIGHT = [((28, 4), 128, 1, 64, 700, True), ((8, 2), 128, 9, 16, 64, True), ((4, 2), 128, 40, 16, 100, True), ((28, 4), 128, 37, 64, 257, True),
         ((6, 1), 64, 90, 32, 511, True), ((8, 2), 128, 70, 128, 300, False), ((40, 1), 64, 2, 16, 77, True), ((3, 3), 128, 260, 64, 300, True)]


@pytest.mark.parametrize("shape", TIGHT, ids=str)
def test_sums_of_bf16_attention_are_fp32_sums(shape):
    """Products of bf16 numbers are exact in fp32: log-sum-exps and weights, which are never rounded to bf16, keep to the bars of fp32."""
    heads, D, n, page_rows, end, causal = shape
    rng = np.random.default_rng(end + 1)
    (H, Hkv), ends = heads, [[end - 3 * g for g in range(heads[1])]]
    cache = Cache(rng, 1, Hkv, -(-end // page_rows), page_rows, D, BF16)
    cache.poison(ends)
    Q = rand(rng, 1, H, n, D, dtype=BF16) * 2
    desc = ob.make_chunk_desc(Q, n_kv_heads=Hkv, causal=causal)
    acc = torch.rand(1, Hkv, cache.cap, device="cuda")
    before = host(acc)
    with np.errstate(invalid="ignore"):
        pool = cache.oracle()
        O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints(ends), ints([n]), acc_in=acc, acc_out=acc)
        wO, wl, ww, pv, qk = po.attend(host(Q), pool, np.array(ends), [n], causal, float(np.float32(desc.softmax_scale)))
    _, el, ew = attend_bars(Q, pool, F32, 0, wO, wl, pv, qk, ww, before, H // Hkv, n)
    dead = np.isneginf(wl)
    assert np.array_equal(np.isneginf(host(lse)), dead)
    within(host(lse)[~dead], wl[~dead], el[~dead], "lse")
    for g in range(Hkv):
        within(host(acc)[0, g, :ends[0][g]], (before + ww)[0, g, :ends[0][g]], ew[0, g, :ends[0][g]], "weights")


# ------------------------------------------------------------------ eviction

def border_weights(rng, kind, n, border):
    if kind == "spread":
        return (border * (1 + 1e-3 * rng.standard_normal(n))).astype(np.float32)
    low, close = {"few": (200, 100), "many": (200, 200)}[kind]
    w = np.full(n, border, dtype=np.float32)
    w[:low] = 0.97 * border
    w[low:low + close] = np.nextafter(np.float32(border), np.float32(0))
    return w[rng.permutation(n)]


@pytest.mark.parametrize("rows,pages", [(2300, 36), (4096, 64), (7000, 128), (8192, 128), (12000, 256), (16384, 256), (17000, 266)])
@pytest.mark.parametrize("kind", ["few", "many", "spread"])
def test_eviction_cuts_below_a_border_of_the_bins(rows, pages, kind):
    """Weights on both sides of a step of a key's upper 11 bits (the pairs' are 0.875 and 1), the cut a few rows off the number of
    those above it; pools of every way to hold the keys."""
    rng = np.random.default_rng(rows)
    cache = Cache(rng, 1, 2, pages, 64, 64, BF16)
    acc = np.stack([np.concatenate([border_weights(rng, kind, rows, b), np.zeros(cache.cap - rows, np.float32)]) for b in (0.875, 1.0)])
    acc = torch.from_numpy(acc[None]).cuda()
    pos = torch.arange(cache.cap, device="cuda").int().expand(1, 2, -1).contiguous()
    above = int((acc[0, 1, :rows] >= 1).sum())
    for i, budget in enumerate((above - 1, above, above + 1, above + 50, above + 101)):
        check_eviction(cache, budget, 0, 0, [cache.cap + 1], [[rows, rows]], pos.clone(), acc.clone(), i % 2 == 0)


@pytest.mark.parametrize("pages", [128, 256, 257])
def test_eviction_below_a_border_stays_inside_its_scratch(pages):
    """Few rows leave from among many: what is listed has to be no more than what moves."""
    rng = np.random.default_rng(pages)
    cache, ws = Cache(rng, 1, 2, pages, 64, 64, BF16), Guarded()
    n = cache.cap
    acc = torch.from_numpy(np.stack([border_weights(rng, "many", n, 1.0) for _ in range(2)])[None]).cuda()
    pos = torch.arange(n, device="cuda").int().expand(1, 2, -1).contiguous()
    for budget in (n - 300, n - 399, n - 350):
        outs = [torch.full((2 * n + 256,), -7, dtype=dt, device="cuda") for dt in (torch.int32, torch.float32)]
        ob.omni_paged_evict(cache.pool, budget, 0, 0, ints([n + 1]), ints([[n, n]]), pos, acc, ws=ws,
                            row_pos_out=outs[0][:-256].view(1, 2, n), acc_out=outs[1][:-256].view(1, 2, n))
        ws.check()
        assert all((x[-256:] == -7).all() for x in outs)


# ------------------------------------------------------------------ the binding

def test_the_short_ways_to_stream_and_device_are_the_public_ones():
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            assert ob._raw_stream(0) == torch.cuda.current_stream().cuda_stream == stream.cuda_stream
            assert ob._current_device() == torch.cuda.current_device()
