"""What attention keeps of small and large values, of probabilities far below the largest, of infinities and of extreme logits, on every kind of launch: rows of
up to 16, 32, 64, 128 and more queries.

Tolerances.  u = 2^-24; E, the error of a logit's exponent to base 2, is at most (2 D + 8) u c sum|q||k| with c = log2(e) / sqrt(D): two roundings a term,
and the products of 16-bit values are exact in fp32.  Softmax numerators and their sum are each off by ln 2 E + 2^-22 relative (exp2 included), sums of n terms by
(n / 16 + 64) u (partial sums of at least 16 lanes), a probability that is split into two values of the type by half a step of half a step, 2^-16 in bf16 and
2^-22 in fp16, all relative to sum p|v|; in fp16, where the largest
probability of a share is at least 2^11 and the smallest step 2^-24, by at least 2^-36 of the largest one, times the largest value.  Out adds its own rounding, half a step (of fp16 below 2^-14 half of 2^-24)."""
import math

import pytest
import torch

import oracle
from paper_2605_16360_amd import binding as pk
from paper_2605_16360_amd import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, HF = torch.bfloat16, torch.float16
# (query heads, new tokens): rows of 4, 16, 20, 52, 120, 132 and 520 queries, which every kind of launch is among
QUERIES = [(4, 1), (4, 4), (4, 5), (4, 13), (8, 15), (4, 33), (8, 65)]


@pytest.fixture(scope="module")
def ctx():
    c = pk.proxykv_create(pk.config_for_case(synth.CASES["tiny"]))
    yield c
    torch.cuda.synchronize()
    pk.proxykv_destroy(c)


def _randn(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def _bounds(q, k, v, lens, exact=False):
    """(out, weight) of the oracle and what each may be off by, without any allowance that is not relative to what is summed.
    exact: logits far from zero that fp32 sums hold.  A difference of two is exact, its exponent (at most 2^7 where it counts) rounded once, and so is a log-sum-exp
    of less than 2^12: ln 2 times 2^-17, and 2^-13 of a probability in the account."""
    rows, G, T, D = q.shape
    out, w, _, spread = oracle.attend(q[None], k[None], v[None], lens[None])
    n = k.shape[1]
    mass = (q.double().abs().reshape(rows, G * T, D) @ k.double().abs().transpose(1, 2)).amax((1, 2)).view(rows, 1, 1, 1)
    rel = 2 * (math.log(2) * (2 * D + 8) * U * 1.4427 / math.sqrt(D) * mass + 2.0 ** -22) + (n / 16 + 64) * U
    if exact:
        rel = torch.full_like(rel, 2 * (2.0 ** -17 + 2.0 ** -22) + (n / 16 + 64) * U)
    half = torch.finfo(q.dtype).eps / 2
    split = half ** 2 * 1.01
    least = 2.0 ** -25 + n * 2.0 ** -36 * float(v.abs().max()) if q.dtype == HF else 0.0
    tol_out = spread[0] * (rel + split) + half * (1 + 2.0 ** -8) * out[0].abs() + least
    tol_w = w[0] * (rel[:, 0, 0] + (2.0 ** -13 if exact else 0) + (G * T + 2) * U) + G * T * 2.0 ** -126  # (fp32 has no full precision below 2^-126: the smallest of each query's terms may be lost)
    return out[0], tol_out, w[0], tol_w


def _within(got, ref, tol, name):
    g = got.double().cpu()
    assert bool(torch.isfinite(g).all()), f"{name}: not finite"
    err = (g - ref).abs()
    assert bool((err <= tol).all()), f"{name}: worst {float((err / tol.clamp_min(1e-300)).max()):.3g} of the bound, max abs err {float(err.max()):.3e}"


def _attend(ctx, q, k, v, lens=None, account=True, exact=False):
    lens = torch.full((k.shape[0],), k.shape[1], dtype=torch.int32) if lens is None else torch.tensor(lens, dtype=torch.int32)
    w = torch.zeros(k.shape[:2], device="cuda") if account else None
    out = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), v.cuda(), lens=lens.cuda(), weight=w)
    torch.cuda.synchronize()
    ref, tol, w_ref, w_tol = _bounds(q, k, v, lens, exact)
    _within(out, ref, tol, "out")
    if account:
        _within(w, w_ref, w_tol, "weight")


# ---- the bits of values and of probabilities ------------------------------------------------------------------------

@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype,scale", [(BF, 1e-8), (BF, 2.0 ** -60), (BF, 2.0 ** 60), (HF, 2.0 ** -12), (HF, 2.0 ** 12)])
def test_values_of_every_size_are_kept(ctx, G, T, dtype, scale):
    """Values that are all small or all large, however many queries there are."""
    for D, N in ((128, 700), (64, 333)):
        _attend(ctx, _randn((2, G, T, D), T, dtype), _randn((2, N, D), T + 1, dtype), _randn((2, N, D), T + 2, dtype, scale), [N, N - 70])


@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype,scale", [(BF, 2.0 ** 127), (HF, 2.0 ** 15)])
@pytest.mark.parametrize("N", [130, 3000, 20000])
def test_the_largest_values_that_there_are(ctx, G, T, dtype, scale, N):
    """Values near the type's largest, all of one sign: their average is finite, and so is everything on the way to it."""
    v = ((1.0 + 0.9 * torch.rand(1, N, 64, generator=torch.Generator().manual_seed(N))) * scale).to(dtype)
    _attend(ctx, _randn((1, G, T, 64), 1, dtype, 0.0 if T % 2 else 2.0), _randn((1, N, 64), 2, dtype), v)


@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_probabilities_are_not_one_16_bit_value(ctx, G, T, dtype):
    """Two keys of nearly the same logit with opposite values among keys without any: out is the difference of two probabilities, to the bits of both."""
    D, N = 64, 192
    q = torch.zeros(2, G, T, D)
    q[..., 0], q[..., 1] = 2.0, _randn((2, G, T), 3, dtype).float() * 0.01
    k = torch.zeros(2, N, D)
    k[:, 5, 0] = k[:, 70, 0] = 4.0
    k[:, 70, 1] = 4.0
    v = torch.zeros(2, N, D)
    v[:, 5], v[:, 70] = 1.0, -1.0
    _attend(ctx, q.to(dtype), k.to(dtype), v.to(dtype), account=False)


@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("above", [12, 17, 24])
def test_what_lies_far_below_a_sink(ctx, G, T, dtype, above):
    """A first key that takes nearly all of the weight and has no value: out is what is left of the others, `above` nats below it."""
    for D, N in ((128, 1100), (64, 2000)):
        q, k, v = _randn((2, G, T, D), above, dtype), _randn((2, N, D), above + 1, dtype), _randn((2, N, D), above + 2, dtype, 1024.0)
        q[..., 0], k[:, :, 0], v[:, 0] = 4.0, 0.0, 0.0
        k[:, 0] = 0.0
        k[:, 0, 0] = above * math.sqrt(D) / 4
        _attend(ctx, q, k, v, [N, N - 333])


@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [8.0, 60.0])
def test_sharp_logits_and_references_that_move(ctx, G, T, dtype, scale):
    """Logits of standard deviations up to 60, and the same growing along the row by as much, so that the largest come last."""
    D, N = 128, 1500
    q, k, v = _randn((2, G, T, D), 5, dtype, scale), _randn((2, N, D), 6, dtype), _randn((2, N, D), 7, dtype)
    q[..., 0] = scale
    k[1, :, 0] = torch.linspace(0, 50, N).to(dtype)
    _attend(ctx, q, k, v, [N - 200, N])


# ---- logits far from zero -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,a,b", [(BF, 1, 3), (BF, 4, 5), (BF, 10, 12), (BF, 20, 25), (BF, 55, 60), (HF, 3, 4), (HF, 13, 12)])
def test_logits_far_from_zero(ctx, G, T, dtype, a, b, sign):
    """Logits that are whole multiples of 2^(a + b), up to 2^123 and down to -2^123, which fp32 sums hold exactly: the largest have all of the weight, in equal
    shares.  Every third query is small and has ordinary ones."""
    for D, N in ((128, 700), (64, 333)):
        g = torch.Generator().manual_seed(a + b)
        q, k = torch.randint(-1, 2, (2, G, T, D), generator=g).float(), torch.randint(-1, 2, (2, N, D), generator=g).float()
        q[..., :D // 2], k[..., :D // 2] = 2.0 * sign, 2.0
        q, k = q * 2.0 ** a, k * 2.0 ** b
        q.view(2, G * T, D)[:, ::3] *= 2.0 ** (-a - b - 4)
        q, k, v = q.to(dtype), k.to(dtype), _randn((2, N, D), a, dtype)
        for account in (True, False):
            _attend(ctx, q, k, v, [N, N - 70], account, exact=True)


# ---- values that are not finite -------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 128), (BF, 64), (HF, 64)])
@pytest.mark.parametrize("N,at", [(700, 0), (700, 300), (700, 690), (70, 3), (2100, 1030)])
def test_infinite_values(ctx, G, T, dtype, D, N, at):
    """A value of plus or minus infinity is that in every output that sees it, wherever it lies; both, or a NaN, are a NaN; all other outputs and the account are
    as they are without it."""
    inf, nan = float("inf"), float("nan")
    q, k, v = _randn((2, G, T, D), 5, dtype), _randn((2, N, D), 6, dtype), _randn((2, N, D), 7, dtype)
    lens = torch.tensor([N, N - 1], dtype=torch.int32)
    bad = v.clone()
    bad[0, at, 3], bad[0, at, 9], bad[0, at, 20] = inf, -inf, nan
    bad[0, at, 33], bad[0, at + 1, 33] = inf, -inf
    w = torch.zeros(2, N, device="cuda")
    out = pk.proxykv_attend(ctx, q.cuda(), k.cuda(), bad.cuda(), lens=lens.cuda(), weight=w)
    torch.cuda.synchronize()
    ref, tol, w_ref, w_tol = _bounds(q, k, v, lens)
    got = out.double().cpu()
    sees = [(torch.arange(T) + N - T >= x).expand(G, T) for x in (at, at + 1)]
    for d, hit in ((3, inf), (9, -inf)):
        assert bool((got[0, :, :, d][sees[0]] == hit).all()), d
    assert bool(got[0, :, :, 20][sees[0]].isnan().all()) and bool(got[0, :, :, 33][sees[1]].isnan().all())
    assert bool((got[0, :, :, 33][sees[0] & ~sees[1]] == inf).all())
    for d in (3, 9, 20, 33):
        got[0, :, :, d][sees[0]] = ref[0, :, :, d][sees[0]]
    _within(got, ref, tol, "out")
    _within(w, w_ref, w_tol, "weight")


@pytest.mark.parametrize("B,T", [(1, 1), (7, 1), (12, 1), (40, 1), (20, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_infinite_shared_values(ctx, B, T, dtype):
    """The same among the shared tokens, in front of every sequence's own."""
    H, G, D, P, N = 2, 4, 128, 900, 150
    q, ks, vs = _randn((B, H, G, T, D), 1, dtype), _randn((H, P, D), 2, dtype), _randn((H, P, D), 3, dtype)
    k, v = _randn((B, H, N, D), 4, dtype), _randn((B, H, N, D), 5, dtype)
    vs[0, 100, 3], vs[1, 899, 4], v[0, 1, 10, 5] = float("inf"), float("-inf"), float("inf")
    out = pk.proxykv_attend_shared(ctx, q.cuda(), ks.cuda(), vs.cuda(), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    want = torch.zeros(B, H, G, T, D, dtype=torch.float64)
    want[:, 0, ..., 3], want[:, 1, ..., 4], want[0, 1, ..., 5] = float("inf"), float("-inf"), float("inf")
    got = out.double().cpu()
    assert torch.equal(torch.where(got.isfinite(), 0.0, got), want)


@pytest.mark.parametrize("B,T", [(2, 1), (7, 1), (16, 1), (40, 1), (24, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("kind", ["sharp", "sink", "small", "far"])
def test_shared_tokens_in_front_of_own(ctx, B, T, dtype, kind):
    """Rows of 8 to 288 queries on the shared tokens and of 4 and 12 on a sequence's own: logits that grow to the last own token, a shared sink without a value, small
    values, and logits far from zero, of which the own ones are as large as the shared."""
    H, G, D, P, N = 2, 4, 128, 900, 150
    q, k, v = _randn((B, H, G, T, D), B, dtype), _randn((B, H, P + N, D), B + 1, dtype), _randn((B, H, P + N, D), B + 2, dtype)
    if kind == "sharp":
        q = q * 16
        q[..., 0] = 16.0
        k[..., 0] = torch.linspace(0, 50, P + N).to(dtype)
    elif kind == "sink":
        q[..., 0], k[..., 0] = 4.0, 0.0
        k[:, :, 0] = 0.0
        k[:, :, 0, 0] = 17 * math.sqrt(D) / 4
        v = v * 1024
        v[:, :, 0] = 0.0
    elif kind == "small":
        v = v * 2.0 ** (-27 if dtype == BF else -10)
    else:
        g = torch.Generator().manual_seed(B)
        q, k = torch.randint(-1, 2, q.shape, generator=g).float(), torch.randint(-1, 2, k.shape, generator=g).float()
        q[..., :64], k[..., :64] = -2.0, 2.0
        q, k = (q * 2.0 ** 12).to(dtype), (k * 2.0 ** 12).to(dtype)
    k[:, :, :P], v[:, :, :P] = k[:1, :, :P], v[:1, :, :P]
    ks, vs, ko, vo = (x.contiguous().cuda() for x in (k[0, :, :P], v[0, :, :P], k[:, :, P:], v[:, :, P:]))
    w, ws = torch.zeros(B, H, N, device="cuda"), torch.zeros(H, P, device="cuda")
    out = pk.proxykv_attend_shared(ctx, q.cuda(), ks, vs, ko, vo, weight_shared=ws, weight=w)
    torch.cuda.synchronize()
    ref_ws, tol_ws = torch.zeros(H, P, dtype=torch.float64), torch.zeros(H, P, dtype=torch.float64)
    for b in range(B):
        ref, tol, w_ref, w_tol = _bounds(q[b], k[b], v[b], torch.full((H,), P + N, dtype=torch.int32), exact=kind == "far")
        _within(out[b], ref, tol, "out")
        _within(w[b], w_ref[:, P:], w_tol[:, P:], "weight")
        ref_ws += w_ref[:, :P]
        tol_ws += w_tol[:, :P]
    _within(ws, ref_ws, tol_ws + ref_ws * B * U, "weight_shared")


@pytest.mark.parametrize("G,T", QUERIES)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_the_largest_values_with_logits_far_from_zero(ctx, G, T, dtype):
    """Both extremes at once, with a logit per query that all keys share."""
    N, D = 2000, 64
    q, k = torch.full((1, G, T, D), -2.0 ** 12), torch.full((1, N, D), 2.0 ** 12)
    v = (1.0 + 0.9 * torch.rand(1, N, D, generator=torch.Generator().manual_seed(2))) * 2.0 ** (127 if dtype == BF else 15)
    _attend(ctx, q.to(dtype), k.to(dtype), v.to(dtype), exact=True)
