"""Decoding on the compacted cache, called through the C ABI, against the 64-bit oracle: attention of new tokens with its account of
weights, the same for a batch on a shared context, eviction by that account, and a run of them behind the path that fills the cache.

Tolerances.  u = 2^-24.  A logit is a sum of D products of 16-bit values, which fp32 holds exactly; counting two roundings a term, its exponent to
base 2 is off by at most E = (2 D + 8) u c sum|q||k| with c = log2(e) / sqrt(D).  Softmax numerators and their sum are each off by ln 2 E + 2^-22 relative
(exp2 included), sums of n terms by another (n / 16 + 64) u (partial sums of at least 16 lanes), a probability split into two 16-bit values by
2^-16, in fp16 by at least 2^-25 of the largest one; with more than 128 queries a row and bf16 values, one rounded to fp16 by half its step, 2^-12.  out is off by that, relative to sum p|v|, and by its own rounding, half a step; weight by the
same relative to what is added, the number of its terms times u, and its own rounding."""
import math

import pytest
import torch

import oracle
from paper_2605_16360_amd import binding as pk
from paper_2605_16360_amd import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, HF = torch.bfloat16, torch.float16
SENTINEL = -7.25


@pytest.fixture(scope="module")
def ctx():
    c = pk.proxykv_create(pk.config_for_case(synth.CASES["tiny"]))
    yield c
    torch.cuda.synchronize()
    pk.proxykv_destroy(c)


def _randn(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def _check(got, got_w, got_ws, q, k, v, lens, w0, ks=None, vs=None, slens=None, ws0=None):
    """Compares with the oracle, under the bound of the module's head."""
    B, H, G, T, D = q.shape
    out, w, ws, spread = oracle.attend(q, k, v, lens, ks, vs, slens)
    N, P = k.shape[2], 0 if ks is None else ks.shape[1]
    c = 1.4427 / math.sqrt(D)
    rel = torch.zeros(B, H)
    most_v = torch.zeros(B, H)
    for b in range(B):
        for h in range(H):
            n = N if lens is None else min(max(int(lens[b][h]), 0), N)
            m = 0 if not P else P if slens is None else min(max(int(slens[h]), 0), P)
            keys = torch.cat([k[b, h, :n]] + ([ks[h, :m]] if m else [])).double().abs()
            vals = torch.cat([v[b, h, :n]] + ([vs[h, :m]] if m else [])).double().abs()
            if keys.shape[0] == 0:
                continue
            E = (2 * D + 8) * U * c * float((q[b, h].reshape(G * T, D).double().abs() @ keys.T).max())
            queries = G * T * (B if m else 1)     # of the row, or of the shared tokens
            rel[b, h] = 2 * (math.log(2) * E + 2.0 ** -22) + ((n + m) / 16 + 64) * U + (2.0 ** -12 if q.dtype == BF and queries > 128 else 2.0 ** -16)
            most_v[b, h] = float(vals.max()) * (n + m) * 2.0 ** -25
    g = got.double().cpu()
    assert bool(torch.isfinite(g).all()), "non-finite output"
    half = torch.finfo(q.dtype).eps / 2
    tol = spread * rel[:, :, None, None, None] + half * (1 + 2.0 ** -8) * out.abs() + (most_v[:, :, None, None, None] if q.dtype == HF else 0) + 2.0 ** -25
    err = (g - out).abs()
    assert bool((err <= tol).all()), f"out: worst {float((err / tol).max()):.3g} of the bound, max abs err {float(err.max()):.3e}"
    for name, a, ref, a0, r in (("weight", got_w, w, w0, rel[:, :, None]), ("weight_shared", got_ws, ws, ws0, rel.max(0).values[:, None])):
        if a is None:
            continue
        terms = G * T * (B if name == "weight_shared" else 1)
        x, x0 = a.double().cpu(), a0.double()
        tol = ref * (r + terms * U) + 2 * U * (x0.abs() + ref) + 1e-30
        err = (x - x0 - ref).abs()
        assert bool((err <= tol).all()), f"{name}: worst {float((err / tol).max()):.3g} of the bound, max abs err {float(err.max()):.3e}"


def _spoil(k, v, w, lens):
    """What lies behind the rows: NaN and infinities, and a value in the account that has to stay."""
    k, v = k.clone(), v.clone()
    rows, N = k.shape[:-2].numel(), k.shape[-2]
    for r in range(rows):
        n = min(max(int(lens.reshape(-1)[r]), 0), N)
        kk, vv = k.view(rows, N, -1)[r], v.view(rows, N, -1)[r]
        kk[n:], vv[n:] = float("nan"), float("inf")
        vv[n::2] = float("nan")
        if w is not None:
            w.view(rows, N)[r, n:] = SENTINEL
    return k, v


def _attend(ctx, rows, G, T, N, D, dtype, lens, seed, scale=1.0, weight=True):
    q, k, v = _randn((rows, G, T, D), seed, dtype, scale), _randn((rows, N, D), seed + 1, dtype), _randn((rows, N, D), seed + 2, dtype)
    lens = torch.tensor(lens, dtype=torch.int32)
    w0 = torch.rand(rows, N, generator=torch.Generator().manual_seed(seed + 3)) if weight else None
    kb, vb = _spoil(k, v, w0, lens)
    w = w0.cuda() if weight else None
    out = pk.proxykv_attend(ctx, q.cuda(), kb.cuda(), vb.cuda(), lens=lens.cuda(), weight=w)
    torch.cuda.synchronize()
    if weight:
        for r in range(rows):
            n = min(max(int(lens[r]), 0), N)
            assert bool((w.cpu()[r, n:] == SENTINEL).all())
    _check(out[None], w[None] if weight else None, None, q[None], k[None], v[None], lens[None], w0[None] if weight else None)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (HF, 128), (HF, 64)])
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000])
def test_attend_lengths(ctx, dtype, D, N):
    """Rows of no token, one, one less than all, all, and lengths outside the row, which count as its ends."""
    _attend(ctx, 7, 4, 1, N, D, dtype, [0, 1, N - 1, N, N // 2, N + 5, -3], seed=N)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("G,T", [(1, 1), (3, 1), (7, 1), (8, 2), (16, 1), (17, 1), (4, 5), (5, 3), (1, 33), (33, 1), (2, 32), (4, 16), (3, 43), (1, 129), (5, 52), (8, 40)])
def test_attend_queries(ctx, dtype, D, G, T):
    """Query tiles that are cut, filled, and one more; the new tokens see different lengths, and some rows have fewer than T."""
    N = 333
    _attend(ctx, 5, G, T, N, D, dtype, [N, max(T - 1, 0), T, 0, 200], seed=G * 100 + T)


@pytest.mark.parametrize("rows,G,T,N", [(1, 4, 1, 70001), (3, 7, 1, 20011), (2, 4, 130, 4099), (1, 1, 300, 300), (300, 1, 1, 33), (1, 64, 1, 9000)])
def test_attend_long_rows_and_many(ctx, rows, G, T, N):
    """Rows that several workgroups share, more rows than the chip has compute units, a whole sequence at once."""
    lens = [N - (r * 37) % (N // 2 + 1) for r in range(rows)]
    _attend(ctx, rows, G, T, N, 128, BF, lens, seed=N, weight=N < 30000)
    _attend(ctx, rows, G, T, N, 64, HF, lens, seed=N + 50)


@pytest.mark.parametrize("rows,G,T,N", [(256, 4, 1, 512), (257, 4, 1, 512), (256, 1, 1, 1), (257, 2, 3, 40), (9, 4, 1, 511), (9, 4, 1, 512), (9, 4, 1, 513), (9, 16, 1, 512),
                                        (9, 17, 1, 512), (9, 2, 8, 513), (9, 1, 1, 545), (9, 4, 4, 640)])
def test_attend_few_keys_and_one_more(ctx, rows, G, T, N):
    """Rows that one workgroup takes from beginning to end, and what is a row, a query or a token more than that; empty rows among them."""
    lens = [0 if r % 5 == 3 else N - (r * 37) % (N // 2 + 1) for r in range(rows)]
    _attend(ctx, rows, G, T, N, 128, BF, lens, seed=N + rows)
    _attend(ctx, rows, G, T, N, 64, HF, lens, seed=N + rows + 9, weight=False)


@pytest.mark.parametrize("scale", [0.0, 8.0, 60.0])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attend_flat_and_sharp_logits(ctx, scale, dtype):
    """All logits equal, and logits of standard deviation up to 60, far above those of the first tiles in later ones."""
    _attend(ctx, 3, 4, 3, 1500, 128, dtype, [1500, 1111, 40], seed=int(scale), scale=scale)


def test_attend_without_lens_and_without_weight(ctx):
    q, k, v = _randn((2, 4, 1, 128), 1, BF), _randn((2, 77, 128), 2, BF), _randn((2, 77, 128), 3, BF)
    out = torch.empty(2, 4, 1, 128, dtype=BF, device="cuda")
    r = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), v.cuda(), out=out)
    torch.cuda.synchronize()
    assert r.data_ptr() == out.data_ptr()
    _check(out[None], None, None, q[None], k[None], v[None], None, None)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T,N", [(4, 100), (40, 64), (40, 300)])
def test_attend_tokens_that_only_later_queries_see(ctx, bad, T, N):
    """NaN and infinities in the last token's key and value reach the last query and none in front of it, in out and in the account."""
    for dtype, D in ((BF, 128), (HF, 64)):
        q, k, v = _randn((2, 3, T, D), 5, dtype), _randn((2, N, D), 6, dtype), _randn((2, N, D), 7, dtype)
        kb, vb = k.clone(), v.clone()
        kb[:, N - 1], vb[:, N - 1] = bad, bad
        w = torch.zeros(2, N, device="cuda")
        out = pk.proxykv_attend(ctx, q.cuda(), kb.cuda(), vb.cuda(), weight=w)
        first = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), vb.cuda())   # the value alone is bad
        torch.cuda.synchronize()
        assert not bool(torch.isfinite(first[:, :, T - 1]).any())
        assert bool(torch.isfinite(first[:, :, :T - 1]).all()) and bool(torch.isfinite(out[:, :, :T - 1]).all())
        qs = q[:, :, :T - 1].contiguous()
        # (in the oracle the last query is left out, so that its row ends one token earlier)
        for o in (out, first):
            _check(o[None, :, :, :T - 1], None, None, qs[None], k[None, :, :N - 1], v[None, :, :N - 1], None, None)


def test_attend_beyond_two_to_the_31_elements(ctx):
    """The last row of a cache of 2.5e9 elements, which starts behind 32-bit offsets."""
    rows, N, D = 64, 300001, 128
    k, v = torch.empty(rows, N, D, dtype=BF, device="cuda"), torch.empty(rows, N, D, dtype=BF, device="cuda")
    kl, vl = _randn((1, 700, D), 1, BF), _randn((1, 700, D), 2, BF)
    k[-1, :700], v[-1, :700] = kl.cuda()[0], vl.cuda()[0]
    lens = torch.zeros(rows, dtype=torch.int32)
    lens[-1] = 700
    q = _randn((rows, 4, 1, D), 3, BF)
    w = torch.zeros(rows, N, device="cuda")
    out = pk.proxykv_attend(ctx, q.cuda(), k, v, lens=lens.cuda(), weight=w)
    torch.cuda.synchronize()
    assert not bool(out[:-1].any()) and not bool(w[:-1].any()) and not bool(w[-1, 700:].any())
    _check(out[None, -1:], w[None, -1:, :700], None, q[None, -1:], kl[None], vl[None], None, torch.zeros(1, 1, 700))
    # the whole of the last row: its own end
    k[-1, N - 700:], v[-1, N - 700:] = kl.cuda()[0], vl.cuda()[0]
    k[-1, :N - 700] = 0
    k[-1, :N - 700, 0] = -100.0
    q[-1, :, :, 0] = 100.0                                # everything but the last 700 has logits of about -880
    kl2 = kl.clone()
    lens[-1] = N
    v[-1, :N - 700] = 0
    out = pk.proxykv_attend(ctx, q.cuda(), k, v, lens=lens.cuda())
    torch.cuda.synchronize()
    _check(out[None, -1:], None, None, q[None, -1:], kl2[None], vl[None], None, None)


# ---- a batch on a shared context ------------------------------------------------------------------------------------

def _shared(ctx, B, H, G, T, P, N, D, dtype, slens, lens, seed, scale=1.0):
    q = _randn((B, H, G, T, D), seed, dtype, scale)
    ks, vs = _randn((H, P, D), seed + 1, dtype), _randn((H, P, D), seed + 2, dtype)
    slens = torch.tensor(slens, dtype=torch.int32)
    ws0 = torch.rand(H, P, generator=torch.Generator().manual_seed(seed + 3))
    ksb, vsb = _spoil(ks, vs, ws0, slens)
    ws = ws0.cuda()
    if N == 0:
        k = v = torch.zeros(B, H, 0, D, dtype=dtype)
        out = pk.proxykv_attend_shared(ctx, q.cuda(), ksb.cuda(), vsb.cuda(), shared_lens=slens.cuda(), weight_shared=ws)
        torch.cuda.synchronize()
        return _check(out, None, ws, q, k, v, None, None, ks, vs, slens, ws0)
    k, v = _randn((B, H, N, D), seed + 4, dtype), _randn((B, H, N, D), seed + 5, dtype)
    lens = torch.tensor(lens, dtype=torch.int32).view(B, H)
    w0 = torch.rand(B, H, N, generator=torch.Generator().manual_seed(seed + 6))
    kb, vb = _spoil(k, v, w0, lens)
    w = w0.cuda()
    out = pk.proxykv_attend_shared(ctx, q.cuda(), ksb.cuda(), vsb.cuda(), kb.cuda(), vb.cuda(), shared_lens=slens.cuda(), lens=lens.cuda(),
                                   weight_shared=ws, weight=w)
    torch.cuda.synchronize()
    for h in range(H):
        assert bool((ws.cpu()[h, min(max(int(slens[h]), 0), P):] == SENTINEL).all())
    _check(out, w, ws, q, k, v, lens, w0, ks, vs, slens, ws0)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("B,G,T,P,N", [(1, 1, 1, 1, 1), (1, 4, 1, 100, 7), (2, 4, 1, 31, 33), (3, 7, 1, 257, 64), (5, 4, 2, 1000, 40), (17, 1, 1, 64, 16),
                                       (16, 4, 1, 513, 20), (33, 4, 1, 200, 5), (65, 4, 1, 300, 3), (4, 8, 9, 129, 30), (2, 4, 1, 8191, 500)])
def test_attend_shared(ctx, dtype, D, B, G, T, P, N):
    """Query tiles of every size, heads with all shared tokens, some and none, sequences with all own tokens, some and none."""
    H = 3
    lens = [(N * (i % 4)) // 3 if i % 4 else 0 for i in range(B * H)]
    _shared(ctx, B, H, G, T, P, N, D, dtype, [P, P // 2, 0], lens, seed=B * 1000 + P)


@pytest.mark.parametrize("B,G,P", [(1, 4, 50), (9, 4, 700), (40, 4, 1500)])
def test_attend_shared_without_own_tokens(ctx, B, G, P):
    _shared(ctx, B, 2, G, 1, P, 0, 128, BF, [P, P - 3], None, seed=P)
    _shared(ctx, B, 2, G, 3, P, 0, 64, HF, [P, 1], None, seed=P)


def test_attend_shared_sharp_logits(ctx):
    _shared(ctx, 6, 2, 4, 2, 900, 70, 128, BF, [900, 451], [70, 3, 2, 0, 69, 70, 1, 70, 33, 32, 31, 64], seed=4, scale=20.0)


def test_attend_shared_is_attend_on_the_joined_cache(ctx):
    """The shared tokens copied in front of every sequence's own give the same, up to the rounding of out and the order of sums."""
    B, H, G, D, P, N = 5, 2, 4, 128, 640, 48
    q, ks, vs = _randn((B, H, G, 1, D), 1, BF).cuda(), _randn((H, P, D), 2, BF).cuda(), _randn((H, P, D), 3, BF).cuda()
    k, v = _randn((B, H, N, D), 4, BF).cuda(), _randn((B, H, N, D), 5, BF).cuda()
    a = pk.proxykv_attend_shared(ctx, q, ks, vs, k, v)
    b = pk.proxykv_attend(ctx, q, torch.cat([ks.expand(B, H, P, D), k], 2), torch.cat([vs.expand(B, H, P, D), v], 2))
    torch.cuda.synchronize()
    assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -8 * float(b.abs().max())


# ---- eviction -------------------------------------------------------------------------------------------------------

def _evict(ctx, rows, N, D, lens, budget, recent, seed, dtype=BF, positions=True, budgets=None, w=None):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randint(-30000, 30000, (rows, N, D), generator=g, dtype=torch.int16).view(dtype) for _ in range(2))
    if w is None:
        w = torch.rand(rows, N, generator=g)
        w[1::3] = torch.round(w[1::3] * 4) / 4
        w[2::6] = 0.5
        w[3::6, ::2] = float("nan")
        w[4::6] = torch.where(w[4::6] < 0.3, -0.0, w[4::6])
        w[5::6, ::3] = float("inf")
        w[5::6, 1::3] = float("-inf")
    pos = torch.randint(0, 1 << 30, (rows, N), generator=g, dtype=torch.int32) if positions else None
    lens_t = torch.tensor(lens, dtype=torch.int32)
    b = budgets if budgets is not None else [budget] * rows
    dev = [x.cuda() if x is not None else None for x in (k, v, w, pos, lens_t)]
    pk.proxykv_evict(ctx, dev[0], dev[1], dev[2], dev[4], torch.tensor(budgets, dtype=torch.int32).cuda() if budgets is not None else budget, recent,
                     positions=dev[3])
    torch.cuda.synchronize()
    source, new = oracle.evict(w, lens, b, recent)
    assert dev[4].tolist() == new
    wide = source.unsqueeze(-1).expand(rows, N, D)
    for got, x in ((dev[0], k), (dev[1], v)):
        assert torch.equal(got.cpu().view(torch.int16), torch.gather(x.view(torch.int16), 1, wide))
    assert torch.equal(dev[2].cpu().view(torch.int32), torch.gather(w, 1, source).view(torch.int32))
    if positions:
        assert torch.equal(dev[3].cpu(), torch.gather(pos, 1, source))


@pytest.mark.parametrize("N,budget,recent", [(1, 1, 0), (2, 1, 1), (2, 1, 0), (65, 64, 0), (65, 64, 64), (257, 256, 31), (1000, 333, 100), (1000, 999, 998), (1025, 1, 0),
                                             (2051, 1024, 1000), (5000, 2500, 7), (5000, 4999, 2000), (9001, 300, 299)])
def test_evict_bit_exact(ctx, N, budget, recent):
    """Ties, NaN, infinities and both zeros in the account; rows that are full, one over the budget, at it, below it, empty, and of lengths outside."""
    lens = [N, N, N, N, N, N, min(budget + 1, N), budget, budget - 1, 0, N + 9, -4]
    _evict(ctx, 12, N, 128, lens, budget, recent, seed=N + budget)


@pytest.mark.parametrize("D,dtype", [(8, BF), (24, HF), (64, HF), (72, BF), (256, BF)])
def test_evict_widths(ctx, D, dtype):
    _evict(ctx, 6, 700, D, [700, 699, 500, 350, 351, 700], 350, 90, seed=D, dtype=dtype, positions=D != 64)


def test_evict_budgets_of_their_own(ctx):
    """Budgets of every row, from below the recent tokens to beyond the row."""
    _evict(ctx, 8, 800, 128, [800, 800, 800, 700, 700, 64, 65, 800], None, 64, seed=3, budgets=[100, 64, 3, 699, 700, 64, 64, 5000])


def test_evict_to_nothing_and_nothing_but_the_recent(ctx):
    """Budgets of no token, of fewer than none, of one, and of the recent tokens alone."""
    _evict(ctx, 6, 90, 64, [90, 90, 1, 0, 90, 2], None, 0, seed=8, budgets=[0, -7, 0, 0, 1, 1])
    _evict(ctx, 3, 90, 64, [90, 41, 40], 40, 40, seed=9)
    _evict(ctx, 3, 2100, 64, [2100, 1300, 1299], 1300, 1300, seed=10)


@pytest.mark.parametrize("rows,N,budget,recent", [(2, 40000, 30000, 500), (1, 170000, 51000, 1024), (300, 600, 580, 128), (3, 36864, 36863, 0), (2, 36865, 20000, 20000)])
def test_evict_long_rows_and_many(ctx, rows, N, budget, recent):
    _evict(ctx, rows, N, 64, [N - (r % 7) for r in range(rows)], budget, recent, seed=N)


def test_evict_narrow_range_of_weights(ctx):
    """Weights that share their high digits, and rows in which every candidate is equal or NaN."""
    w = torch.rand(4, 4000, generator=torch.Generator().manual_seed(1)) * 1e-4 + 0.25
    w[1] = 3.0
    w[2] = float("nan")
    w[3] = float("-inf")
    _evict(ctx, 4, 4000, 64, [4000, 4000, 4000, 3999], 3000, 17, seed=5, w=w)


@pytest.mark.parametrize("N", [1500, 12000, 45000])
@pytest.mark.parametrize("same,bits", [(255, 21), (256, 21), (257, 21), (256, 10), (257, 10), (600, 10)])
def test_evict_keys_that_agree_in_front(ctx, N, same, bits):
    """The weight that decides is among `same` ones that differ in their last `bits` bits at most, some of them equal, as many as are ranked by comparison
    and one more; the budget ends at the first, the last, and in between."""
    g = torch.Generator().manual_seed(same + bits)
    rows, w = 6, torch.rand(6, N, generator=g) * 0.5
    w[:, ::2] += 2.0                                        # half above, half below the ones that agree, near 1.0
    for r in range(rows):
        at = torch.randperm(N - 5, generator=g)[:same]
        low = torch.randint(0, 1 << bits, (same,), generator=g, dtype=torch.int32)
        low[:5] = low[0]
        w[r, at] = (low + 0x3f800000).view(torch.float32)
    heavy = [int((w[r, :N - 5] >= 2).sum()) for r in range(rows)]
    budgets = [5 + heavy[0] + 1, 5 + heavy[1] + same, 5 + heavy[2] + same // 2, 5 + heavy[3] + 3, 5 + heavy[4], 5 + heavy[5] + same + 1]
    _evict(ctx, rows, N, 8, [N] * rows, None, 5, seed=N + same, budgets=budgets, w=w)


def test_evict_beyond_two_to_the_31_elements(ctx):
    rows, N, D = 64, 300001, 128
    k, v = torch.empty(rows, N, D, dtype=BF, device="cuda"), torch.empty(rows, N, D, dtype=BF, device="cuda")
    kl, vl = _randn((N, D), 1, BF).cuda(), _randn((N, D), 2, BF).cuda()
    k[-1], v[-1] = kl, vl
    w = torch.zeros(rows, N, device="cuda")
    w[-1] = torch.rand(N, generator=torch.Generator().manual_seed(3)).cuda()
    w_last = w[-1].cpu()
    lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    lens[-1] = N
    pk.proxykv_evict(ctx, k, v, w, lens, 200000, 1000)
    torch.cuda.synchronize()
    source, new = oracle.evict(w_last[None], [N], [200000], 1000)
    assert lens.tolist() == [0] * 63 + [200000]
    at = source[0].cuda()
    assert torch.equal(k[-1], kl[at]) and torch.equal(v[-1], vl[at]) and torch.equal(w[-1].cpu(), w_last[source[0]])


# ---- as they are used -----------------------------------------------------------------------------------------------

def test_same_bits_every_time_and_on_another_stream(ctx):
    """Calls back to back, on a stream of their own, and of two contexts on two streams at once."""
    q, k, v = _randn((24, 4, 2, 128), 1, BF).cuda(), _randn((24, 3001, 128), 2, BF).cuda(), _randn((24, 3001, 128), 3, BF).cuda()
    lens = torch.tensor([3001 - 100 * i for i in range(24)], dtype=torch.int32, device="cuda")
    w = [torch.zeros(24, 3001, device="cuda") for _ in range(4)]
    ref = pk.proxykv_attend(ctx, q, k, v, lens=lens, weight=w[0])
    again = pk.proxykv_attend(ctx, q, k, v, lens=lens, weight=w[1])
    torch.cuda.synchronize()
    other = pk.proxykv_create(ctx.cfg)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a = pk.proxykv_attend(ctx, q, k, v, lens=lens, weight=w[2], stream=s1)
    b = pk.proxykv_attend(other, q, k, v, lens=lens, weight=w[3], stream=s2)
    torch.cuda.synchronize()
    pk.proxykv_destroy(other)
    for x, y in ((again, w[1]), (a, w[2]), (b, w[3])):
        assert torch.equal(x.view(torch.int16), ref.view(torch.int16)) and torch.equal(y, w[0])


def test_calls_in_a_graph(ctx):
    """A decoding step and an eviction captured once and replayed with new contents, eager calls of the same context in between, and
    every replay equal to the eager result; a context without the workspace refuses and leaves the capture whole."""
    rows, G, N, D, budget, recent = 6, 4, 2001, 128, 1900, 50
    q, k, v = (torch.zeros(rows, *s, D, dtype=BF, device="cuda") for s in ((G, 1), (N,), (N,)))
    lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    w, out = torch.zeros(rows, N, device="cuda"), torch.zeros(rows, G, 1, D, dtype=BF, device="cuda")

    def fill(seed):
        q.copy_(_randn(q.shape, seed, BF))
        k.copy_(_randn(k.shape, seed + 1, BF))
        v.copy_(_randn(v.shape, seed + 2, BF))
        lens.copy_(torch.tensor([N, N - 3, 1900, 1901, 7, 0], dtype=torch.int32))
        w.zero_()

    def step():
        pk.proxykv_attend(ctx, q, k, v, lens=lens, weight=w, out=out)
        pk.proxykv_evict(ctx, k, v, w, lens, budget, recent)

    fill(0)
    step()
    torch.cuda.synchronize()
    small = pk.proxykv_create(ctx.cfg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(pk.ProxyKVError) as e:
            pk.proxykv_evict(small, k, v, w, lens, budget, recent)
        assert e.value.status == pk.PROXYKV_ESTATE
        with pytest.raises(pk.ProxyKVError) as e:
            pk.proxykv_attend(small, q, k, v, lens=lens, weight=w, out=out)
        assert e.value.status == pk.PROXYKV_ESTATE
        step()
    pk.proxykv_destroy(small)
    for seed in (10, 20, 30):
        fill(seed)
        step()
        torch.cuda.synchronize()
        ref = [x.clone() for x in (out, k, v, w, lens)]
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, k, v, w, lens), ref):
            assert torch.equal(x, y)


@pytest.mark.parametrize("B,H,G,T,P,N,D,dtype", [(1, 6, 4, 1, 0, 300, 128, BF), (1, 3, 4, 5, 0, 900, 64, HF), (1, 2, 4, 70, 0, 1100, 128, BF), (1, 2, 3, 16, 0, 777, 64, BF),
                                                  (3, 2, 4, 1, 800, 40, 128, BF), (40, 2, 4, 1, 900, 33, 128, BF), (5, 2, 4, 1, 700, 64, 64, HF)])
def test_every_kind_of_launch_in_a_graph(ctx, B, H, G, T, P, N, D, dtype):
    """One launch and several, kept logits and those that are computed again, in parts and not: three replays on new contents, eager calls of the same context in
    front of each, equal to those bit for bit."""
    q, out = (torch.zeros(B, H, G, T, D, dtype=dtype, device="cuda") for _ in range(2))
    k, v = (torch.zeros(B, H, N, D, dtype=dtype, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(H, max(P, 1), D, dtype=dtype, device="cuda") for _ in range(2))
    w, ws = torch.zeros(B, H, N, device="cuda"), torch.zeros(H, max(P, 1), device="cuda")
    lens = torch.tensor([[N - (b * H + h) % 7 for h in range(H)] for b in range(B)], dtype=torch.int32, device="cuda")

    def fill(seed):
        for i, x in enumerate((q, k, v, ks, vs)):
            x.copy_(_randn(x.shape, seed + i, dtype))
        w.fill_(0.5)
        ws.zero_()

    def step():
        if P:
            pk.proxykv_attend_shared(ctx, q, ks, vs, k, v, lens=lens, weight_shared=ws, weight=w, out=out)
        else:
            pk.proxykv_attend(ctx, q, k, v, lens=lens, weight=w, out=out)

    fill(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (10, 20, 30):
        fill(seed)
        step()
        torch.cuda.synchronize()
        ref = [x.clone() for x in (out, w, ws)]
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, w, ws), ref):
            assert torch.equal(x, y)


@pytest.mark.parametrize("pooled", [False, True])
def test_prune_then_decode_and_evict(ctx, pooled):
    """The path as a program runs it: a context is selected and compacted where it lies, with a budget per head or per layer, tokens are
    decoded on it one at a time with an account, the cache is cut back every eight tokens, and decoding goes on.  A plain copy
    of cache and account is kept with the oracle; the selection of every eviction is that of the account that the library kept."""
    L, H, G, N, K, D, recent, steps = 2, 3, 4, 400, 150, 128, 16, 21
    k, v = _randn((L, H, N, D), 1, BF).cuda(), _randn((L, H, N, D), 2, BF).cuda()
    scores = _randn((L, H, N), 3, torch.float32).cuda()
    if pooled:
        flat, counts = pk.proxykv_topk_pooled(ctx, scores, K)
        pk.proxykv_compact_pooled(ctx, k, v, flat, counts)
        lens, budgets = counts.clone(), counts.clone()
    else:
        pk.proxykv_compact_inplace(ctx, k, v, pk.proxykv_topk(ctx, scores, K))
        lens, budgets = torch.full((L, H), K, dtype=torch.int32, device="cuda"), None
    weight = torch.zeros(L, H, N, device="cuda")
    positions = torch.arange(N, dtype=torch.int32, device="cuda").expand(L, H, N).contiguous()
    for step in range(steps):
        for l in range(L):
            kn, vn, q = (_randn(s, 100 + 10 * step + l + i, BF).cuda() for i, s in enumerate(((H, 1, D), (H, 1, D), (H, G, 1, D))))
            at = lens[l].long().view(H, 1)
            k[l].scatter_(1, at[:, :, None].expand(H, 1, D), kn)
            v[l].scatter_(1, at[:, :, None].expand(H, 1, D), vn)
            weight[l].scatter_(1, at, 0.0)
            positions[l].scatter_(1, at, N + step)
            lens[l] += 1
            w0 = weight[l].cpu().clone()
            out = pk.proxykv_attend(ctx, q, k[l], v[l], lens=lens[l], weight=weight[l])
            torch.cuda.synchronize()
            _check(out[None], weight[None, l], None, q[None].cpu(), k[None, l].cpu(), v[None, l].cpu(), lens[None, l].cpu(), w0[None])
        if step % 8 == 7:
            before = [x.cpu().clone() for x in (k, v, weight, positions, lens)]
            pk.proxykv_evict(ctx, k, v, weight, lens, budgets if pooled else K, recent, positions=positions)
            torch.cuda.synchronize()
            b = (budgets.cpu().view(-1).tolist() if pooled else [K] * (L * H))
            source, new = oracle.evict(before[2].view(L * H, N), before[4].view(-1).tolist(), b, recent)
            assert lens.view(-1).tolist() == new
            source = source.view(L, H, N)
            assert torch.equal(weight.cpu(), torch.gather(before[2], 2, source)) and torch.equal(positions.cpu(), torch.gather(before[3], 2, source))
            for x, y in ((k, before[0]), (v, before[1])):
                assert torch.equal(x.cpu(), torch.gather(y, 2, source.unsqueeze(-1).expand(L, H, N, D)))


def test_prune_then_share(ctx):
    """A context is compacted out of place by the fused call and then serves a batch as the shared tokens, whose account decides what of
    it is evicted; decoding goes on with what is left."""
    case = synth.CASES["tiny"]
    w = synth.make_mapper_weights(case.H_kv, case.H_l)
    c = pk.proxykv_create(pk.config_for_case(case))
    pk.proxykv_set_mapper_weights(c, w)
    q, kc, kr = (x.cuda() for x in synth.make_proxy_qk(case))
    kt, vt = (x.cuda() for x in synth.make_target_kv(case))
    ks, vs, idx, K = pk.proxykv_prune(c, q, kc, kr, case.chunk, 0.3, kt, vt)
    B, H, G, D, N = 6, case.H_l, 4, case.D, 20
    shared, shared_v, slens = ks[0], vs[0], torch.full((H,), K, dtype=torch.int32, device="cuda")
    account, positions = torch.zeros(H, K, device="cuda"), idx[0].clone()
    for step, budget in ((0, K - 40), (1, K - 70)):
        qd, k, v = _randn((B, H, G, 1, D), step, BF).cuda(), _randn((B, H, N, D), step + 10, BF).cuda(), _randn((B, H, N, D), step + 20, BF).cuda()
        lens = torch.full((B, H), N - 1 + step, dtype=torch.int32, device="cuda")
        a0, s0, l0 = account.cpu().clone(), [x.cpu().clone() for x in (shared, shared_v)], slens.cpu().clone()
        out = pk.proxykv_attend_shared(c, qd, shared, shared_v, k, v, shared_lens=slens, lens=lens, weight_shared=account)
        torch.cuda.synchronize()
        _check(out, None, account, qd.cpu(), k.cpu(), v.cpu(), lens.cpu(), None, s0[0], s0[1], l0, a0)
        a1, p1 = account.cpu().clone(), positions.cpu().clone()
        pk.proxykv_evict(c, shared, shared_v, account, slens, budget, 0, positions=positions)
        torch.cuda.synchronize()
        source, new = oracle.evict(a1, l0.tolist(), [budget] * H, 0)
        assert slens.tolist() == new
        assert torch.equal(positions.cpu(), torch.gather(p1, 1, source))
        assert torch.equal(shared.cpu(), torch.gather(s0[0], 1, source.unsqueeze(-1).expand(H, K, D)))
    pk.proxykv_destroy(c)


@pytest.mark.parametrize("far", [0, 70, 200, 511, 900])
def test_attend_many_queries_with_values_beyond_half(ctx, far):
    """Blocks of many queries multiply bf16 values as half: values up to 65 280 and tiny ones as they are, and from the first key with one of
    65 536 or more (up to 2^100, or not finite) on, another way; outputs that do not meet it are as near as any."""
    G, T, N, D = 8, 40, 1001, 128
    q, k, v = _randn((2, G, T, D), 5, BF), _randn((2, N, D), 6, BF), _randn((2, N, D), 7, BF)
    v[0, far, ::2], v[1, far, 1::3] = 65280.0, 2.0 ** -30
    v[1, :, 5] *= 2.0 ** -12
    lens = torch.tensor([N, N - 1], dtype=torch.int32)
    w0 = torch.zeros(2, N)
    for big in (None, 65536.0, 2.0 ** 100):
        if big is not None:
            v[0, far, 7], v[1, far, 0] = big, -big
        w = w0.cuda()
        out = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), v.cuda(), lens=lens.cuda(), weight=w)
        torch.cuda.synchronize()
        _check(out[None], w[None], None, q[None], k[None], v[None], lens[None], w0[None])
    v[0, far, 7] = float("inf")
    out = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), v.cuda(), lens=lens.cuda())
    torch.cuda.synchronize()
    assert not bool(torch.isfinite(out[0, :, :, 7]).any())
    keep = [i for i in range(D) if i != 7]
    assert bool(torch.isfinite(out[0][..., keep]).all()) and bool(torch.isfinite(out[1]).all())
