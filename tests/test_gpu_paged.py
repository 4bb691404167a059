"""Rotary positions and the paged cache against the 64-bit oracle, through the public binding."""
import itertools

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2511_12201_amd import binding as ob

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24                          # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def rand(rng, *shape, dtype=F32):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def within(got, want, bar, what=""):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want)
    bad = ~(np.abs(got - want) <= bar) & ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.where(bad, np.abs(got - want), 0))} "
                           f"at {np.argwhere(bad)[0]}, allowed {np.broadcast_to(bar, bad.shape)[tuple(np.argwhere(bad)[0])]}")


# ------------------------------------------------------------------ rotary positions

def rope_bar(x, want, rot, interleaved, dtype):
    """A turned element is u c - v s: the angle's fraction of a turn is rounded to 32 bits (at most 2^-26 turns = 2^-23.3
    radians), sine and cosine are off by two steps (2^-22 of 1) and the three operations by one half step each; then it is
    stored.  Together under 8e-7 (|u| + |v|)."""
    pair = np.abs(x).astype(np.float64)
    head = pair[..., :rot]
    mates = (head.reshape(*head.shape[:-1], -1, 2)[..., ::-1].reshape(head.shape) if interleaved
             else np.roll(head, rot // 2, axis=-1))
    reach = np.concatenate([head + mates, np.zeros_like(pair[..., rot:])], -1)
    return 8e-7 * reach * 1.01 + half_step(dtype) * np.abs(want) * (dtype is BF16)


def layer(Q, K):
    return ob.make_layer_desc(Q, K, 0, Q.shape[2])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,batch", [(1, (4, 2), 2), (37, (7, 1), 1), (130, (28, 4), 2)])
def test_rope_forward_and_backward(dtype, D, rot, interleaved, n, heads, batch):
    rng = np.random.default_rng(n + rot)
    plan = ob.make_rope_desc(D, rot, interleaved=interleaved, base=1e5, scaling="by_parts", factor=4.0, orig_len=2048)
    f = po.rope_frequencies(rot, 1e5, "by_parts", 4.0, 2048)
    Q, K = rand(rng, batch, heads[0], n, D, dtype=dtype), rand(rng, batch, heads[1], n, D, dtype=dtype)
    pos = rng.integers(-1000, 1 << 20, (batch, n)).astype(np.int32)
    for backward, sign in ((False, 1.0), (True, -1.0)):
        out = ob.omni_rope(plan, layer(Q, K), Q, K, torch.from_numpy(pos).cuda(), backward=backward)
        for x, got in zip((Q, K), out):
            want = po.rope(host(x), pos[:, None], f, interleaved, sign)
            within(host(got), want, rope_bar(host(x), want, rot, interleaved, dtype), f"backward {backward}")
            assert torch.equal(got[..., rot:], x[..., rot:])


def test_rope_default_positions_in_place_strided_and_scaled():
    rng = np.random.default_rng(3)
    base = rand(rng, 2, 19, 6, 64, dtype=BF16)                       # tokens before heads, and a gap behind the keys
    Q, K = base[:, :, :4].transpose(1, 2), base[:, :, 4:5].transpose(1, 2)
    keep = base.clone()
    plan = ob.make_rope_desc(64, 32, out_scale=1.25)
    d = layer(Q, K)
    Qn, Kn = ob.omni_rope(plan, d, Q, K)
    assert Qn.stride() == Q.stride() and torch.equal(base, keep)
    f = po.rope_frequencies(32)
    want = po.rope(host(Q), np.arange(19), f, False, 1.0, 1.25)
    within(host(Qn), want, 1.25 * rope_bar(host(Q), want, 32, False, BF16))
    assert ob.omni_rope(plan, d, Q, K, Qout=Q, Kout=K)[0] is Q
    assert torch.equal(Q, Qn) and torch.equal(K, Kn)
    assert torch.equal(base[:, :, 5], keep[:, :, 5])                 # what lies between the rows stays


def test_rope_gradient_is_the_difference_quotient_of_the_forward_pass():
    """The map is linear: <dy, f(x + h e) - f(x)> / h for a step that the sums hold exactly, against the gradient."""
    rng = np.random.default_rng(4)
    plan = ob.make_rope_desc(64, 64, interleaved=True)
    Q, K = rand(rng, 1, 2, 5, 64), rand(rng, 1, 1, 5, 64)
    dQ, dK = rand(rng, 1, 2, 5, 64), rand(rng, 1, 1, 5, 64)
    pos = ints([[0, 1, 77, 4000, 900001]])
    gQ, gK = ob.omni_rope(plan, layer(Q, K), dQ, dK, pos, backward=True)
    y = ob.omni_rope(plan, layer(Q, K), Q, K, pos)[0]
    for at in itertools.product([0, 1], [1, 4], [0, 7, 63]):
        X = Q.clone()
        X[0][at] += 4.0
        diff = host(ob.omni_rope(plan, layer(X, K), X, K, pos)[0]) - host(y)
        step = float(X[0][at].double() - Q[0][at].double())
        # two forward passes, each off by 8e-7 (|u| + |v|) < 8e-6 in the two elements of the pair
        assert abs((host(dQ) * diff).sum() / step - float(gQ[0][at])) < 4 * 8e-6 * 4 / step + 1e-5
    # and the adjoint as a whole: <dy, R x> = <R^T dy, x>
    a, b = (host(dQ) * host(y)).sum(), (host(gQ) * host(Q)).sum()
    assert abs(a - b) < 8e-7 * 4 * np.abs(host(dQ)).sum() * np.abs(host(Q)).max()


def test_rope_surrounds_the_training_calls():
    """Q, K turned, attention forward and backward on full lists, gradients turned back: against float64 autograd of the whole."""
    rng = np.random.default_rng(5)
    N, H, D = 48, 4, 64
    Q, K, V, dO = (rand(rng, 1, h, N, D) for h in (H, 2, 2, H))
    plan, desc = ob.make_rope_desc(D, 32), ob.make_layer_desc(Q, K, 0, 40)
    pos = ints([list(range(500, 500 + N))])
    Qr, Kr = ob.omni_rope(plan, desc, Q, K, pos)
    full = torch.arange(N, dtype=torch.int32, device="cuda").expand(1, H, N).contiguous()
    cnt, budget = torch.full((1, H), N, dtype=torch.int32, device="cuda"), ints([N])
    O, lse = ob.omni_sparse_attn_fwd(desc, Qr, Kr, V, full, cnt, full, budget, N)
    dQ, dK, dV = ob.omni_sparse_attn_bwd(desc, Qr, Kr, V, O, dO, lse, full, cnt, full, budget, N)
    dQ, dK = ob.omni_rope(plan, desc, dQ, dK, pos, backward=True, Qout=dQ, Kout=dK)

    q, k, v = (x.double().cpu().requires_grad_() for x in (Q, K, V))
    f = torch.from_numpy(po.rope_frequencies(32))
    a = torch.arange(500, 500 + N).double()[:, None] * f
    turn = lambda x: torch.cat([x[..., :16] * a.cos() - x[..., 16:32] * a.sin(), x[..., :16] * a.sin() + x[..., 16:32] * a.cos(),  # noqa: E731
                                x[..., 32:]], -1)
    z = turn(q) @ turn(k).repeat_interleave(2, 1).transpose(-1, -2) / 8
    z = z.masked_fill(torch.triu(torch.ones(N, N, dtype=torch.bool), 1), -float("inf"))
    o = z.softmax(-1) @ v.repeat_interleave(2, 1)
    o.backward(dO.double().cpu())
    within(host(O), o.detach().numpy(), 1e-4)                       # the library's bar for fp32
    for got, leaf in ((dQ, q), (dK, k), (dV, v)):
        within(host(got), leaf.grad.numpy(), 1e-4)


# ------------------------------------------------------------------ the paged cache

class Cache:
    """A pool, its table and what the rows carry, on the GPU and as the oracle holds it."""

    def __init__(self, rng, B, Hkv, pages, page_rows, D, dtype, fill=None):
        total = B * Hkv * pages
        self.K, self.V = (rand(rng, total + 2, page_rows, D, dtype=dtype) for _ in range(2))
        self.table = torch.from_numpy(rng.permutation(total + 2)[:total].reshape(B, Hkv, pages).astype(np.int32)).cuda()
        self.cap = pages * page_rows
        self.page_rows = page_rows

    @property
    def pool(self):
        return ob.make_page_pool(self.K, self.V, self.table)

    def oracle(self):
        return po.Pool(host(self.K), host(self.V), self.table.cpu().numpy())

    def poison(self, row_end, value=float("nan")):
        """Everything that is no row in use: rows behind the ends, pages in nobody's table."""
        B, Hkv, pages = self.table.shape
        used = torch.zeros(self.K.shape[:2], dtype=torch.bool)
        table = self.table.cpu()
        for b, g in itertools.product(range(B), range(Hkv)):
            for j in range(min(max(int(row_end[b][g]), 0), self.cap)):
                page = int(table[b, g, j // self.page_rows])
                if 0 <= page < len(used):
                    used[page, j % self.page_rows] = True
        self.K[~used.cuda()] = value
        self.V[~used.cuda()] = value


def attend_bars(Q, pool, dtype, scale, O, lse, pv, qk, weights, acc, G, n):
    """fp32 products and sums in any order: a score is off by eS = (D + 2) u qk, a weight by that and a few steps more (2^-21:
    the exponent's product and 2^x), numerator and sum alike, the sums over the rows by rows * u at most.  bf16: every weight of
    the second product is rounded (2^-8 at most), the sum may hold it rounded or not, and the output is stored."""
    D, rows = Q.shape[-1], pool.cap
    e = 2 * ((D + 2) * U32 * qk + 2.0 ** -21) + 2 * rows * U32
    e_o = e[..., None] * pv + (2 * 2.0 ** -8 * pv * 1.01 + 2.0 ** -8 * np.abs(O) if dtype is BF16 else U32 * np.abs(O))
    e_l = e + 4 * U32 * np.abs(lse) + (2.0 ** -8 if dtype is BF16 else 0)
    e_w = None
    if weights is not None:
        top = e.max() + 4 * U32 * np.abs(np.where(np.isfinite(lse), lse, 0)).max()
        e_w = (top + (2.0 ** -8 if dtype is BF16 else 0) + G * n * U32) * weights + 2 * U32 * np.abs(acc + weights)
    return e_o, e_l, e_w


def check_attention(cache, Q, row_end, new_cnt, causal, weights, dtype, desc=None, stream=None):
    B, H, n, D = Q.shape
    Hkv = cache.table.shape[1]
    G = H // Hkv
    desc = desc or ob.make_chunk_desc(Q, n_kv_heads=Hkv, causal=causal)
    acc = torch.rand(B, Hkv, cache.cap, device="cuda") if weights else None
    out = torch.full_like(acc, -7.0) if weights else None
    O = ob._like(Q, (*desc.q_stride, 1)).fill_(float("nan"))
    lse = torch.full((B, H, n), float("nan"), device="cuda")
    ob.omni_paged_attn(desc, Q, cache.pool, ints(row_end), ints(new_cnt), O=O, lse=lse, acc_in=acc, acc_out=out)
    torch.cuda.synchronize()
    scale = float(np.float32(desc.softmax_scale))
    pool = cache.oracle()
    with np.errstate(invalid="ignore"):
        wO, wl, ww, pv, qk = po.attend(host(Q), pool, np.array(row_end), np.array(new_cnt), causal, scale)
    eO, el, ew = attend_bars(Q, pool, dtype, scale, wO, wl, pv, qk, ww if weights else None, host(acc) if weights else None, G, n)
    within(host(O), wO, eO, "O")
    dead = np.isneginf(wl)
    assert np.array_equal(np.isneginf(host(lse)), dead) and not host(O)[dead].any()
    within(host(lse)[~dead], wl[~dead], el[~dead], "lse")
    if weights:
        got, want = host(out), host(acc) + ww
        for b, g in itertools.product(range(B), range(Hkv)):
            end = min(max(int(row_end[b][g]), 0), cache.cap)
            within(got[b, g, :end], want[b, g, :end], ew[b, g, :end], "weights")
            assert (got[b, g, end:] == -7.0).all()
    return O, lse, out


SHAPES = [
    # heads, D, n_new, page_rows, row_end (per pair, varied below), causal
    ((4, 2), 64, 1, 16, 1, True), ((4, 2), 128, 1, 16, 33, True), ((7, 1), 128, 1, 64, 200, True), ((28, 4), 128, 1, 64, 700, True),
    ((2, 2), 64, 3, 32, 3, True), ((8, 2), 128, 9, 16, 64, True), ((21, 3), 64, 5, 32, 65, True), ((8, 8), 64, 2, 16, 129, False),
    ((4, 2), 128, 40, 16, 100, True), ((28, 4), 128, 37, 64, 257, True), ((4, 4), 64, 130, 16, 130, True),
    ((6, 1), 64, 90, 32, 511, True), ((8, 2), 128, 70, 128, 300, False), ((40, 1), 64, 2, 16, 77, True), ((3, 3), 128, 260, 64, 300, True),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_over_pages(shape, weights, dtype):
    heads, D, n, page_rows, end, causal = shape
    rng = np.random.default_rng(end)
    B, (H, Hkv) = 2, heads
    pages = -(-end // page_rows) + 1
    row_end = [[max(n, end - 3 * g) if b == 0 else max(0, end // 2 - g) for g in range(Hkv)] for b in range(B)]
    new_cnt = [n, min(n, max(0, end // 2 - Hkv), (2 * n + 2) // 3)]
    cache = Cache(rng, B, Hkv, pages, page_rows, D, dtype)
    cache.poison(row_end)
    Q = rand(rng, B, H, n, D, dtype=dtype) * 2
    Q[1, :, new_cnt[1]:] = float("nan")
    check_attention(cache, Q, row_end, new_cnt, causal, weights, dtype)


LONG = [
    # heads, D, n_new, page_rows, row_end per sequence, causal: whole tiles, many spans an item, windows of the page table
    ((14, 2), 128, 1, 64, (9000, 4097), True), ((8, 2), 64, 3, 16, (20011, 64), True), ((4, 1), 128, 16, 32, (3000, 2999), False),
    ((14, 2), 128, 100, 64, (4000, 1531), True), ((6, 2), 64, 333, 16, (2222, 900), True), ((4, 1), 128, 24, 16, (70001, 33000), True),
    ((2, 1), 64, 700, 256, (700, 699), True), ((8, 1), 128, 64, 16, (6400, 6401), False), ((32, 1), 64, 9, 32, (5003, 17), True),
    ((8, 4), 128, 2, 64, (99990, 90001), True),              # more than the caches hold: 389 MB in bf16
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_attention_over_long_caches(shape, dtype):
    """The same on the GPU in float64, head by head."""
    heads, D, n, page_rows, ends, causal = shape
    rng = np.random.default_rng(n)
    (H, Hkv), B = heads, 2
    G = H // Hkv
    cache = Cache(rng, B, Hkv, -(-max(ends) // page_rows) + 1, page_rows, D, dtype)
    row_end = [[e - 7 * g if e > n + 7 * Hkv else e for g in range(Hkv)] for e in ends]
    new_cnt = [n, max(1, min(n - 1, ends[1]))]
    cache.poison(row_end)
    Q = rand(rng, B, H, n, D, dtype=dtype) * 2
    acc_in, acc = torch.rand(B, Hkv, cache.cap, device="cuda"), torch.zeros(B, Hkv, cache.cap, device="cuda")
    desc = ob.make_chunk_desc(Q, n_kv_heads=Hkv, causal=causal)
    O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints(row_end), ints(new_cnt), acc_in=acc_in, acc_out=acc)
    for b, g in itertools.product(range(B), range(Hkv)):
        end, cnt = row_end[b][g], new_cnt[b]
        pages = cache.table[b, g, :-(-end // page_rows)].long()
        k, v = (x[pages].reshape(-1, D)[:end].double() for x in (cache.K, cache.V))
        weights = torch.zeros(end, dtype=torch.float64, device="cuda")
        wl, qk, worst = [], [], 0.0
        for i in range(g * G, (g + 1) * G):
            q = Q[b, i, :cnt].double()
            z = q @ k.T * float(np.float32(desc.softmax_scale))
            hidden = torch.arange(end, device="cuda") >= (end - cnt + 1 + torch.arange(cnt, device="cuda"))[:, None] if causal else \
                torch.zeros_like(z, dtype=torch.bool)
            z.masked_fill_(hidden, -torch.inf)
            l = z.logsumexp(-1)
            p = torch.exp(z - torch.where(l > -torch.inf, l, 0.0)[:, None])
            weights += p.sum(0)
            reach = ((q.abs() @ k.abs().T).masked_fill(hidden, 0).amax(-1) * desc.softmax_scale).cpu().numpy()
            pool = type("P", (), {"cap": end})
            eO, el, ew = attend_bars(host(Q[b, i, :cnt]), pool, dtype, 0, host(p @ v), host(l), host(p @ v.abs()), reach, None, None, G, n)
            within(host(O[b, i, :cnt]), host(p @ v), eO, f"O {b} {i}")
            within(host(lse[b, i, :cnt]), host(l), el, f"lse {b} {i}")
            worst = max(worst, (2 * ((D + 2) * U32 * reach + 2.0 ** -21) + 2 * end * U32 + 4 * U32 * np.abs(host(l))).max())
        bar = (worst + (2.0 ** -8 if dtype is BF16 else 0) + G * n * U32) * host(weights) + 2 * U32 * np.abs(host(acc_in[b, g, :end]) + host(weights))
        within(host(acc[b, g, :end]), host(acc_in[b, g, :end]) + host(weights), bar, "weights")
        assert not O[b, :, cnt:].any() and torch.isneginf(lse[b, :, cnt:]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 6, 50])
def test_empty_sequences_counts_out_of_range_and_chunks_longer_than_their_rows(dtype, n):
    rng = np.random.default_rng(n)
    row_end = [[0, 5], [-3, 10 ** 9], [2, n + 1], [20, 7]]
    new_cnt = [n, 1, n, 0]                                    # sequence 2: fewer rows than new tokens, the first see nothing
    cache = Cache(rng, 4, 2, 4, 16, 64, dtype)
    cache.poison(row_end)
    Q = rand(rng, 4, 6, n, 64, dtype=dtype)
    for causal, weights in itertools.product([True, False], [True, False]):
        check_attention(cache, Q, row_end, new_cnt, causal, weights, dtype)
    check_attention(cache, Q, row_end, [n + 5, -4, n, 2 ** 31 - 1], True, True, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 4, 60])
def test_pages_that_are_not_there(dtype, n):
    rng = np.random.default_rng(n)
    cache = Cache(rng, 2, 2, 6, 16, 128, dtype)
    row_end = [[90, 80], [64, 96]]
    for at, value in (((0, 0, 0), -1), ((0, 0, 3), cache.K.shape[0]), ((0, 1, 2), 2 ** 31 - 1), ((1, 1, 5), -2 ** 31)):
        cache.table[at] = value
    cache.table[1, 0] = -1                                    # a pair with nothing at all
    cache.poison(row_end)
    check_attention(cache, rand(rng, 2, 4, n, 128, dtype=dtype), row_end, [n, n], True, True, dtype)
    check_attention(cache, rand(rng, 2, 4, n, 128, dtype=dtype), row_end, [n, n], False, False, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 5, 40, 300])
def test_a_nan_stays_with_the_tokens_that_see_it(dtype, n):
    rng = np.random.default_rng(n)
    cache = Cache(rng, 2, 1, 30, 16, 64, dtype)
    Q = rand(rng, 2, 3, n, 64, dtype=dtype)
    desc, ends, cnt = ob.make_chunk_desc(Q, n_kv_heads=1), ints([[430], [460]]), ints([n, n])
    outs = []
    row = max(430 - 2, 430 - n)                               # the last one or two tokens see it
    for value in (None, float("nan")):
        if value is not None:
            cache.K[cache.table[0, 0, row // 16].long(), row % 16, 5] = value
        acc = torch.zeros(2, 1, cache.cap, device="cuda")
        outs.append((*ob.omni_paged_attn(desc, Q, cache.pool, ends, cnt, acc_out=acc), acc))
    (O, lse, acc), (bad_O, bad_lse, bad_acc) = outs
    clean = row - (430 - n)
    # rows of a wavefront may take another reference value: weights (2^-8 at most) and outputs are rounded anew; sums of 430 rows
    assert not ((O - bad_O)[0, :, :clean].abs() > 4 * 2.0 ** -8 * cache.V.abs().max()).any() and torch.isfinite(bad_O[0, :, :clean]).all()
    assert ((lse - bad_lse)[0, :, :clean].abs() <= 2 * (2 * 430 * U32 + 2.0 ** -20 + 4 * U32 * 64)).all()
    assert bad_O[0, :, clean:].isnan().all() and bad_lse[0, :, clean:].isnan().all() and bad_acc[0, 0, :row + 1].isnan().all()
    for x, y in ((O, bad_O), (lse, bad_lse), (acc, bad_acc)):
        assert torch.equal(x[1], y[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores_and_equal_scores(dtype):
    """One row that takes everything, all rows alike, and scores that rise from tile to tile."""
    rng = np.random.default_rng(8)
    cache = Cache(rng, 1, 1, 20, 16, 64, dtype)
    Q = rand(rng, 1, 4, 3, 64, dtype=dtype)
    cache.K[cache.table[0, 0, 7].long(), 3] = (30 * Q[0, 0, 0]).to(dtype)
    check_attention(cache, Q, [[310]], [3], True, True, dtype)
    cache.K.zero_()
    check_attention(cache, Q, [[310]], [3], True, True, dtype)
    for page in range(20):
        cache.K[cache.table[0, 0, page].long()] = (0.5 * page * Q[0, 1, 1]).to(dtype)
    check_attention(cache, Q, [[310]], [3], True, True, dtype)
    cache.K[cache.table[0, 0].long()] *= -1
    check_attention(cache, Q, [[310]], [3], False, True, dtype)


def test_strided_chunks_and_a_pool_that_two_sequences_share():
    rng = np.random.default_rng(9)
    cache = Cache(rng, 2, 2, 5, 32, 64, BF16)
    cache.table[1] = cache.table[0]                           # a common prefix, read only
    fused = rand(rng, 2, 11, 8, 64, dtype=BF16)               # [B, tokens, Q heads and K heads, D]
    Q = fused[:, :, :4].transpose(1, 2)
    check_attention(cache, Q, [[140, 150], [77, 160]], [11, 4], True, True, BF16)


def test_a_pool_beyond_four_gigabytes():
    rng = np.random.default_rng(10)
    pages, rows, D = 1 << 17, 256, 128                        # 2^25 rows of 256 bytes each, twice
    K, V = (torch.empty(pages, rows, D, dtype=BF16, device="cuda") for _ in range(2))
    cache = Cache(rng, 1, 1, 2, rows, D, BF16)
    far = ints([[[pages - 1, pages // 2 + 1]]])
    for big, small in ((K, cache.K), (V, cache.V)):
        big[far[0, 0].long()] = small[cache.table[0, 0].long()]
    Q, n = rand(rng, 1, 4, 5, D, dtype=BF16), 300
    desc = ob.make_chunk_desc(Q, n_kv_heads=1)
    a = ob.omni_paged_attn(desc, Q, cache.pool, ints([[n]]), ints([5]))
    b = ob.omni_paged_attn(desc, Q, ob.make_page_pool(K, V, far), ints([[n]]), ints([5]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    rope = ob.make_rope_desc(D)
    new = [rand(rng, 1, h, 5, D, dtype=BF16) for h in (4, 1, 1)]
    pos = torch.zeros(1, 1, 2 * rows, dtype=torch.int32, device="cuda")
    for pool in (cache.pool, ob.make_page_pool(K, V, far)):
        ob.omni_paged_append(ob.make_chunk_desc(new[0], new[1]), rope, *new, pool, ints([n]), ints([5]), ints([[n]]), pos)
    acc = torch.rand(1, 1, 2 * rows, device="cuda")
    for pool in (cache.pool, ob.make_page_pool(K, V, far)):
        ob.omni_paged_evict(pool, 100, 0, 0, ints([10 ** 6]), ints([[n + 5]]), pos, acc)
    for big, small in ((K, cache.K), (V, cache.V)):
        assert torch.equal(big[far[0, 0].long()], small[cache.table[0, 0].long()])


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot", [(64, 32), (128, 128)])
@pytest.mark.parametrize("n", [1, 5, 70])
@pytest.mark.parametrize("turned", [True, False])
def test_append(dtype, D, rot, n, turned):
    rng = np.random.default_rng(n)
    B, H, Hkv = 3, 6, 2
    cache = Cache(rng, B, Hkv, 6, 16, D, dtype)
    cache.table[2, 1, 1] = -1
    cache.table[2, 0, 2] = cache.K.shape[0]
    row_cnt = [[0, 3], [20, 94], [15, 14]]                    # pair (1, 1) runs over its 96 rows
    new_cnt, pos = [n, max(1, n - 2), min(n, 40)], [0, 123456, -5]
    Q, K, V = (rand(rng, B, h, n, D, dtype=dtype) for h in (H, Hkv, Hkv))
    row_pos, acc = torch.full((B, Hkv, cache.cap), -9, dtype=torch.int32, device="cuda"), torch.rand(B, Hkv, cache.cap, device="cuda")
    pool = cache.oracle()
    w_pos, w_acc = row_pos.cpu().numpy(), host(acc)
    freq = po.rope_frequencies(rot, 5e4) if turned else None
    raw = po.Pool(host(cache.K), host(cache.V), cache.table.cpu().numpy())
    po.append(raw, np.stack([host(K)] * 1)[0], host(V), pos, new_cnt, np.array(row_cnt), w_pos.copy(), w_acc.copy())   # unturned
    w_end = po.append(pool, host(K), host(V), pos, new_cnt, np.array(row_cnt), w_pos, w_acc, freq, True)
    plan = ob.make_rope_desc(D, rot, base=5e4, interleaved=True) if turned else None
    before = torch.full_like(Q, 3.0)
    Qout, row_end = ob.omni_paged_append(ob.make_chunk_desc(Q, K), plan, Q if turned else None, K, V, cache.pool, ints(pos),
                                         ints(new_cnt), ints(row_cnt), row_pos, acc=acc, Qout=before if turned else None)
    np.testing.assert_array_equal(row_end.cpu().numpy(), w_end)
    np.testing.assert_array_equal(row_pos.cpu().numpy(), w_pos)
    np.testing.assert_array_equal(host(acc), w_acc)
    np.testing.assert_array_equal(host(cache.V), pool.V)
    if not turned:
        np.testing.assert_array_equal(host(cache.K), pool.K)
        assert Qout is None
        return
    stored = np.any(raw.K != host(torch.zeros(1).cuda()) + pool.K, axis=-1)
    bar = np.where(stored[..., None], rope_bar(raw.K, pool.K, rot, True, dtype), 0)
    within(host(cache.K), pool.K, bar, "K")
    for b in range(B):
        want = po.rope(host(Q)[b, :, :new_cnt[b]], pos[b] + np.arange(new_cnt[b]), freq, True)
        within(host(Qout)[b, :, :new_cnt[b]], want, rope_bar(host(Q)[b, :, :new_cnt[b]], want, rot, True, dtype), "Q")
        assert (Qout[b, :, new_cnt[b]:] == 3.0).all()


@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (128, 128, True), (128, 48, False), (64, 64, True)])
def test_many_rows_are_turned_as_few(D, rot, interleaved):
    """Calls beyond what the caches hold (128 MB in and out) against the same rows in parts, bit for bit."""
    rng = np.random.default_rng(D)
    n, H, Hkv = 16384 * 64 // D + 37, 28, 4
    Q, K, V = (rand(rng, 1, h, n, D, dtype=BF16) for h in (H, Hkv, Hkv))
    plan = ob.make_rope_desc(D, rot, base=1e6, interleaved=interleaved)
    for backward in (False, True):
        q, k = ob.omni_rope(plan, layer(Q, K), Q, K, backward=backward)
        for a in range(0, n, 1500):
            pq, pk = Q[:, :, a:a + 1500].contiguous(), K[:, :, a:a + 1500].contiguous()
            pos = torch.arange(a, a + pq.shape[2], dtype=torch.int32, device="cuda")[None]
            wq, wk = ob.omni_rope(plan, layer(pq, pk), pq, pk, pos, backward=backward)
            assert torch.equal(q[:, :, a:a + 1500], wq) and torch.equal(k[:, :, a:a + 1500], wk)
    one, parts = (Cache(np.random.default_rng(1), 1, Hkv, n // 64 + 1, 64, D, BF16) for _ in range(2))
    row_pos = torch.zeros(1, Hkv, one.cap, dtype=torch.int32, device="cuda")
    q, _ = ob.omni_paged_append(ob.make_chunk_desc(Q, K), plan, Q, K, V, one.pool, ints([7]), ints([n]), ints([[0] * Hkv]), row_pos)
    for a in range(0, n, 1500):
        pq, pk, pv = (x[:, :, a:a + 1500].contiguous() for x in (Q, K, V))
        wq, _ = ob.omni_paged_append(ob.make_chunk_desc(pq, pk), plan, pq, pk, pv, parts.pool, ints([7 + a]), ints([pq.shape[2]]),
                                     ints([[a] * Hkv]), row_pos)
        assert torch.equal(q[:, :, a:a + 1500], wq)
    assert torch.equal(one.K, parts.K) and torch.equal(one.V, parts.V)


def test_append_of_counts_out_of_range():
    rng = np.random.default_rng(2)
    cache = Cache(rng, 3, 1, 2, 16, 64, F32)
    K, V = rand(rng, 3, 1, 4, 64), rand(rng, 3, 1, 4, 64)
    row_pos = torch.zeros(3, 1, 32, dtype=torch.int32, device="cuda")
    pool, w_pos = cache.oracle(), np.zeros((3, 1, 32), dtype=np.int32)
    args = [[1, 2, 3], [-1, 100, 4], np.array([[5], [-8], [1000]])]
    w_end = po.append(pool, host(K), host(V), args[0], args[1], args[2], w_pos, None)
    _, end = ob.omni_paged_append(ob.make_chunk_desc(K, K), None, None, K, V, cache.pool, ints(args[0]), ints(args[1]),
                                  ints(args[2].tolist()), row_pos)
    np.testing.assert_array_equal(end.cpu().numpy(), w_end)
    np.testing.assert_array_equal(row_pos.cpu().numpy(), w_pos)
    np.testing.assert_array_equal(host(cache.K), pool.K)
    np.testing.assert_array_equal(host(cache.V), pool.V)


# ------------------------------------------------------------------ eviction

def check_eviction(cache, budget, sink, recent, seq_len, row_end, row_pos, acc, in_place=False):
    pool = cache.oracle()
    w_cnt, w_pos, w_acc = po.evict(pool, budget, sink, recent, np.array(seq_len), np.array(row_end), row_pos.cpu().numpy(),
                                   acc.cpu().numpy())
    outs = dict(row_pos_out=row_pos, acc_out=acc) if in_place else \
        dict(row_pos_out=torch.full_like(row_pos, -77), acc_out=torch.full_like(acc, -77.0))
    end = ints(row_end)
    cnt, pos, got = ob.omni_paged_evict(cache.pool, budget, sink, recent, ints(seq_len), end, row_pos, acc,
                                        row_cnt=end if in_place else None, **outs)
    np.testing.assert_array_equal(cnt.cpu().numpy(), w_cnt)
    for b, g in itertools.product(*map(range, w_cnt.shape)):
        k = w_cnt[b, g]
        np.testing.assert_array_equal(pos[b, g, :k].cpu().numpy(), w_pos[b, g, :k])
        np.testing.assert_array_equal(got[b, g, :k].cpu().numpy(), w_acc[b, g, :k])
        if not in_place:
            assert (pos[b, g, k:] == -77).all() and (got[b, g, k:] == -77.0).all()
    np.testing.assert_array_equal(host(cache.K), pool.K)
    np.testing.assert_array_equal(host(cache.V), pool.V)


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("budget", [1, 17, 60, 100, 500])
def test_eviction(dtype, D, in_place, budget):
    rng = np.random.default_rng(budget)
    cache = Cache(rng, 2, 2, 7, 16, D, dtype)
    row_end = [[112, 61], [0, 33]]
    acc = torch.from_numpy(rng.exponential(1.0, (2, 2, cache.cap)).astype(np.float32)).cuda()
    pos = torch.from_numpy(np.stack([rng.permutation(400)[:cache.cap] for _ in range(4)]).reshape(2, 2, -1).astype(np.int32)).cuda()
    sink, recent = min(2, budget - 1), min(10, max(0, budget - 2))
    check_eviction(cache, budget, sink, recent, [400, 350], row_end, pos, acc, in_place)


@pytest.mark.parametrize("rows,budget", [(1, 1), (2, 1), (1000, 999), (1025, 1024), (5000, 1250), (5000, 4999), (20000, 7000)])
@pytest.mark.parametrize("kind", ["ties", "zeros", "mixed"])
def test_eviction_with_equal_and_odd_weights(rows, budget, kind):
    rng = np.random.default_rng(rows + budget)
    cache = Cache(rng, 1, 2, -(-rows // 64) + 1, 64, 64, BF16)
    acc = rng.integers(0, 5, (1, 2, cache.cap)).astype(np.float32)
    if kind == "zeros":
        acc[:] = np.where(rng.random(acc.shape) < 0.5, 0.0, -0.0)
    if kind == "mixed":
        acc = rng.choice(np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-40, -1e-40, 3.0, 2.5], dtype=np.float32), acc.shape)
    pos = torch.arange(cache.cap, device="cuda").int().expand(1, 2, -1).contiguous()
    check_eviction(cache, budget, 0, 0, [cache.cap + 1], [[rows, rows - 1]], pos, torch.from_numpy(acc).cuda(), True)


@pytest.mark.parametrize("rows", [900, 3001, 8190, 16383, 17000])
@pytest.mark.parametrize("near", [1, 700, 5000, 1 << 21])
def test_eviction_between_weights_that_are_close(rows, near):
    """`near` neighbouring floats from 1 on, zeros and a few others: cuts in every third of a key, among many equal keys and few."""
    rng = np.random.default_rng(rows + near)
    cache = Cache(rng, 1, 1, -(-rows // 64), 64, 64, BF16)
    acc = (np.float32(1.0).view(np.int32) + rng.integers(0, near, cache.cap).astype(np.int32)).view(np.float32)
    other = rng.random(cache.cap)
    acc = np.where(other < 0.1, np.float32(0.0), np.where(other > 0.99, np.float32(50.0) + other.astype(np.float32), acc))[None, None]
    pos = torch.arange(cache.cap, device="cuda").int()[None, None]
    for budget in (1, rows // 200 + 1, rows // 2, rows - rows // 10 + 3, rows - 1):
        check_eviction(cache, budget, 0, 0, [cache.cap + 1], [[rows]], pos.clone(), torch.from_numpy(acc).cuda(), budget % 2 == 0)


@pytest.mark.parametrize("pages,rows,budget", [(256, 16384, 16383), (256, 16000, 4000), (257, 16448, 100), (257, 300, 299), (257, 0, 5),
                                               (2000, 128000, 32000), (2000, 127999, 127998), (64, 4096, 1), (65, 4097, 4000)])
@pytest.mark.parametrize("kind", ["weights", "zeros"])
def test_eviction_of_long_caches(pages, rows, budget, kind):
    rng = np.random.default_rng(rows)
    cache = Cache(rng, 2, 1, pages, 64, 64, BF16)
    acc = np.exp(2.5 * rng.standard_normal((2, 1, cache.cap))).astype(np.float32) if kind == "weights" else np.zeros((2, 1, cache.cap), dtype=np.float32)
    pos = torch.arange(cache.cap, device="cuda").int().expand(2, 1, -1).contiguous()
    sink, recent = min(4, budget - 1), min(64, max(0, budget - 5))
    check_eviction(cache, budget, sink, recent, [rows, rows // 2], [[rows], [rows // 2 + 1]], pos, torch.from_numpy(acc).cuda())


@pytest.mark.parametrize("pages", [8, 1100])
def test_eviction_at_the_ends_of_the_range_of_positions(pages):
    rng = np.random.default_rng(pages)
    cache = Cache(rng, 1, 1, pages, 16, 64, BF16)
    pos = torch.full((1, 1, cache.cap), 5, dtype=torch.int32, device="cuda")
    pos[0, 0, 40], pos[0, 0, 41] = -2 ** 31, 2 ** 31 - 1
    acc = torch.zeros(1, 1, cache.cap, device="cuda")
    acc[0, 0, 50:60] = 1
    for seq_len, rows in ((-2 ** 31, range(20)),              # every position is recent: the first rows stay
                          (2 ** 31 - 1, [40, 41, *range(50, 60), *range(8)])):
        _, got, weights = ob.omni_paged_evict(cache.pool, 20, 1, 19, ints([seq_len]), ints([[cache.cap - 3]]), pos, acc)
        assert sorted(got[0, 0, :20].tolist()) == sorted(pos[0, 0, list(rows)].tolist())
        assert weights[0, 0, :20].sum().item() == acc[0, 0, list(rows)].sum().item()


def test_eviction_where_more_rows_are_spared_than_fit_and_pages_are_missing():
    rng = np.random.default_rng(1)
    cache = Cache(rng, 1, 2, 5, 16, 64, F32)
    cache.table[0, 1, 0] = -1
    cache.table[0, 1, 4] = 2 ** 31 - 1
    pos = torch.zeros(1, 2, cache.cap, dtype=torch.int32, device="cuda")        # every row claims to be the first token
    acc = torch.rand(1, 2, cache.cap, device="cuda")
    check_eviction(cache, 20, 3, 0, [1000], [[70, 80]], pos, acc)
    check_eviction(cache, 20, 0, 0, [1000], [[70, 80]], pos, acc)


# ------------------------------------------------------------------ together

class Loop:
    """A serving loop: append, attend, evict; the same on the oracle's side from what the kernels stored."""

    def __init__(self, dtype, n, budget, B=2, H=6, Hkv=2, D=64):
        self.rng, self.dtype, self.n, self.budget = np.random.default_rng(n), dtype, n, budget
        self.B, self.H, self.Hkv, self.D = B, H, Hkv, D
        self.cache = Cache(self.rng, B, Hkv, 6, 16, D, dtype)
        cap = self.cache.cap
        self.row_cnt, self.row_end = ints([[0] * Hkv] * B), ints([[0] * Hkv] * B)
        self.row_pos, self.acc = torch.zeros(B, Hkv, cap, dtype=torch.int32, device="cuda"), torch.zeros(B, Hkv, cap, device="cuda")
        self.pos, self.new_cnt = ints([0] * B), ints([n] * B)
        self.plan = ob.make_rope_desc(D, 32)
        self.Q, self.K, self.V = (torch.zeros(B, h, n, D, dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))
        self.Qr, self.O = torch.zeros_like(self.Q), torch.zeros_like(self.Q)
        self.lse = torch.zeros(B, H, n, device="cuda")
        self.desc = ob.make_chunk_desc(self.Q, self.K)
        self.ws = ob.Workspace()

    def inputs(self):
        for x in (self.Q, self.K, self.V):
            x.copy_(rand(self.rng, *x.shape, dtype=self.dtype))

    def step(self):
        ob.omni_paged_append(self.desc, self.plan, self.Q, self.K, self.V, self.cache.pool, self.pos, self.new_cnt, self.row_cnt,
                             self.row_pos, acc=self.acc, Qout=self.Qr, row_end=self.row_end)
        ob.omni_paged_attn(self.desc, self.Qr, self.cache.pool, self.row_end, self.new_cnt, O=self.O, lse=self.lse,
                           acc_in=self.acc, acc_out=self.acc, ws=self.ws)
        self.pos.add_(self.new_cnt)
        ob.omni_paged_evict(self.cache.pool, self.budget, 2, 8, self.pos, self.row_end, self.row_pos, self.acc,
                            row_cnt=self.row_cnt, row_pos_out=self.row_pos, acc_out=self.acc, ws=self.ws)

    def state(self):
        return [x.clone() for x in (self.O, self.lse, self.row_cnt, self.row_end, self.row_pos, self.acc, self.cache.K, self.cache.V)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 5, 30])
def test_a_serving_loop_keeps_to_its_budget_and_its_formulas(dtype, n):
    s = Loop(dtype, n, 40)
    held = [[{} for _ in range(s.Hkv)] for _ in range(s.B)]                     # position -> (K, V) as they were stored
    for step in range(6):
        s.inputs()
        acc, first = s.acc.clone(), s.row_cnt.clone()
        end = ints([[0] * s.Hkv] * s.B)
        ob.omni_paged_append(s.desc, s.plan, s.Q, s.K, s.V, s.cache.pool, s.pos, s.new_cnt, s.row_cnt, s.row_pos, acc=s.acc,
                             Qout=s.Qr, row_end=end)
        pool, acc0 = s.cache.oracle(), host(s.acc)
        wO, wl, ww, pv, qk = po.attend(host(s.Qr), pool, end.cpu().numpy(), [n] * s.B, True, float(np.float32(s.desc.softmax_scale)))
        ob.omni_paged_attn(s.desc, s.Qr, s.cache.pool, end, s.new_cnt, O=s.O, lse=s.lse, acc_in=s.acc, acc_out=s.acc)
        eO, el, ew = attend_bars(s.Q, pool, dtype, 0.125, wO, wl, pv, qk, ww, acc0, 3, n)
        within(host(s.O), wO, eO, "O")
        within(host(s.lse), wl, el, "lse")
        within(host(s.acc), acc0 + ww, ew + 1e-30, "acc")
        s.pos.add_(s.new_cnt)
        w_cnt, w_pos, w_acc = po.evict(pool, 40, 2, 8, s.pos.cpu().numpy(), end.cpu().numpy(), s.row_pos.cpu().numpy(), s.acc.cpu().numpy())
        ob.omni_paged_evict(s.cache.pool, 40, 2, 8, s.pos, end, s.row_pos, s.acc, row_cnt=s.row_cnt, row_pos_out=s.row_pos, acc_out=s.acc)
        np.testing.assert_array_equal(s.row_cnt.cpu().numpy(), w_cnt)
        np.testing.assert_array_equal(host(s.cache.K), pool.K)
        for b, g in itertools.product(range(s.B), range(s.Hkv)):
            k = w_cnt[b, g]
            assert k == min(40, (step + 1) * n) and len(set(w_pos[b, g, :k])) == k
            np.testing.assert_array_equal(s.row_pos[b, g, :k].cpu().numpy(), w_pos[b, g, :k])
            np.testing.assert_array_equal(s.acc[b, g, :k].cpu().numpy(), w_acc[b, g, :k])


@pytest.mark.parametrize("n", [1, 12])
def test_a_captured_step_replayed_is_the_eager_step(n):
    eager, graphed = Loop(BF16, n, 40), Loop(BF16, n, 40)
    for s in (eager, graphed):
        s.inputs()
        s.step()                                             # and the workspace exists
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    for _ in range(7):
        for s in (eager, graphed):
            s.inputs()
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)


def test_two_streams_at_once_and_a_stream_that_is_not_the_default():
    loops = [Loop(BF16, 9, 40), Loop(F32, 1, 30)]
    alone = []
    for s in loops:
        t = Loop(s.dtype, s.n, s.budget)
        for _ in range(5):
            t.inputs()
            t.step()
        torch.cuda.synchronize()
        alone.append(t.state())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(loops, streams):
            with torch.cuda.stream(st):
                s.inputs()
                s.step()
    torch.cuda.synchronize()
    for s, want in zip(loops, alone):
        for a, b in zip(s.state(), want):
            assert torch.equal(a, b)


class Guarded(ob.Workspace):
    """Scratch of exactly the size that is asked for, with a pattern behind it."""

    def get(self, call_id, desc, param=0):
        need = ob.workspace_bytes(call_id, desc, param)
        self.whole = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
        return self.whole[:need]

    def check(self):
        assert (self.whole[-4096:] == 0xAB).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,end", [(1, 4000), (4, 700), (5, 100), (40, 3000), (300, 301)])
def test_calls_stay_inside_their_scratch_and_outputs(dtype, n, end):
    rng = np.random.default_rng(n)
    B, H, Hkv, D = 2, 14, 2, 64
    cache = Cache(rng, B, Hkv, -(-end // 16), 16, D, dtype)
    Q = rand(rng, B, H, n, D, dtype=dtype)
    desc, ws = ob.make_chunk_desc(Q, n_kv_heads=Hkv), Guarded()
    rows = B * H * n
    O, lse, acc = (torch.full((size + 256,), 7.0, dtype=dt, device="cuda") for size, dt in
                   ((rows * D, dtype), (rows, F32), (B * Hkv * cache.cap, F32)))
    ob.omni_paged_attn(desc, Q, cache.pool, ints([[end] * Hkv] * B), ints([n] * B), O=O[:-256].view(Q.shape), lse=lse[:-256].view(B, H, n),
                       acc_out=acc[:-256].view(B, Hkv, cache.cap), ws=ws)
    ws.check()
    assert all((x[-256:] == 7.0).all() for x in (O, lse, acc))


@pytest.mark.parametrize("pages", [3, 64, 200, 1030])
def test_eviction_stays_inside_its_scratch(pages):
    rng = np.random.default_rng(pages)
    cache, ws = Cache(rng, 2, 2, pages, 16, 64, BF16), Guarded()
    acc, pos = torch.rand(2, 2, cache.cap, device="cuda"), torch.zeros(2, 2, cache.cap, dtype=torch.int32, device="cuda")
    ob.omni_paged_evict(cache.pool, cache.cap // 2, 0, 0, ints([5, 5]), ints([[cache.cap] * 2] * 2), pos, acc, ws=ws)
    ws.check()


def test_results_repeat_to_the_bit():
    rng = np.random.default_rng(12)
    cache = Cache(rng, 1, 2, 40, 64, 128, BF16)
    Q = rand(rng, 1, 14, 33, 128, dtype=BF16)
    desc = ob.make_chunk_desc(Q, n_kv_heads=2)
    runs = []
    for _ in range(4):
        acc = torch.zeros(1, 2, cache.cap, device="cuda")
        O, lse = ob.omni_paged_attn(desc, Q, cache.pool, ints([[2500, 2560]]), ints([33]), acc_out=acc)
        runs.append((O, lse, acc))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_a_slimmed_store_of_pages_is_read_by_both_decode_calls():
    """Rows that omni_compact_cache_paged stored are what omni_paged_attn attends: one token over all of them equals
    omni_slim_decode_paged of an active head whose group keeps every visual row and has no other."""
    rng = np.random.default_rng(13)
    N, D, H, Hkv = 150, 128, 4, 2
    Kc, Vc = rand(rng, 1, Hkv, N, D, dtype=BF16), rand(rng, 1, Hkv, N, D, dtype=BF16)
    q = rand(rng, 1, H, D, dtype=BF16)
    d = ob.make_decode_desc(q, Kc, 0, N, tau=-1.0)
    grp_idx = torch.arange(N, dtype=torch.int32, device="cuda").expand(1, Hkv, N).contiguous()
    grp_mask, grp_cnt = torch.full_like(grp_idx, 3), torch.full((1, Hkv), N, dtype=torch.int32, device="cuda")
    cache = Cache(rng, 1, Hkv, 10, 16, D, BF16)
    ob.omni_compact_cache_paged(d, Kc, Vc, grp_idx, grp_cnt, cache.pool)
    probe = torch.zeros(1, Hkv, 2, D, device="cuda")
    O1, _ = ob.omni_slim_decode_paged(d, q, Kc, Vc, ints([N]), probe, cache.pool, grp_idx, grp_mask, grp_cnt)
    Q = q[:, :, None]
    O2, _ = ob.omni_paged_attn(ob.make_chunk_desc(Q, n_kv_heads=Hkv), Q, cache.pool, grp_cnt, ints([1]))
    # both round every weight and the output to bf16 (2^-8 each side) and |V| stays below 5
    assert (O1 - O2[:, :, 0]).abs().max() <= 4 * 2 ** -8 * 5
