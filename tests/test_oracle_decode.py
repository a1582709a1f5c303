"""Pins of the decode oracles (CPU only): per-pair loops, library attention, closed forms and invariants; eviction against
its definition token by token."""
import math

import pytest
import torch

import oracle


def test_attend_is_softmax_attention_token_by_token():
    g = torch.Generator().manual_seed(1)
    B, H, G, T, D, N, P = 2, 2, 2, 3, 8, 7, 5
    q, k, v = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((B, H, G, T, D), (B, H, N, D), (B, H, N, D)))
    ks, vs = torch.randn(H, P, D, generator=g, dtype=torch.float64), torch.randn(H, P, D, generator=g, dtype=torch.float64)
    lens, shared_lens = [[7, 4], [2, 0]], [5, 3]
    out, w, ws, spread = oracle.attend(q, k, v, lens, ks, vs, shared_lens)
    w2, ws2 = torch.zeros_like(w), torch.zeros_like(ws)
    for b in range(B):
        for h in range(H):
            for gg in range(G):
                for t in range(T):
                    own = [n for n in range(lens[b][h]) if n <= lens[b][h] - T + t]
                    logits = [float(q[b, h, gg, t] @ ks[h, n]) / math.sqrt(D) for n in range(shared_lens[h])]
                    logits += [float(q[b, h, gg, t] @ k[b, h, n]) / math.sqrt(D) for n in own]
                    z = sum(math.exp(x) for x in logits)
                    probs = [math.exp(x) / z for x in logits]
                    vals = [vs[h, n] for n in range(shared_lens[h])] + [v[b, h, n] for n in own]
                    ref = sum((p * x for p, x in zip(probs, vals)), torch.zeros(D, dtype=torch.float64))
                    assert torch.allclose(out[b, h, gg, t], ref, rtol=0, atol=1e-12)
                    for n in range(shared_lens[h]):
                        ws2[h, n] += probs[n]
                    for i, n in enumerate(own):
                        w2[b, h, n] += probs[shared_lens[h] + i]
    assert torch.allclose(w, w2, rtol=0, atol=1e-12) and torch.allclose(ws, ws2, rtol=0, atol=1e-12)
    assert bool((spread >= out.abs() - 1e-12).all())


def test_attend_matches_library_attention_and_sums_to_the_queries():
    g = torch.Generator().manual_seed(2)
    q, k, v = torch.randn(1, 2, 3, 4, 16, generator=g), torch.randn(1, 2, 9, 16, generator=g), torch.randn(1, 2, 9, 16, generator=g)
    out, w, none, _ = oracle.attend(q, k, v)
    causal = torch.ones(4, 9, dtype=torch.bool).tril(5)
    for gg in range(3):
        ref = torch.nn.functional.scaled_dot_product_attention(q[0, :, gg].double(), k[0].double(), v[0].double(), attn_mask=causal)
        assert torch.allclose(out[0, :, gg], ref, atol=1e-12)
    assert none is None and torch.allclose(w.sum(-1), torch.full((1, 2), 12.0, dtype=torch.float64))


def test_attend_rows_that_see_nothing():
    q, k = torch.ones(1, 1, 1, 3, 4), torch.ones(1, 1, 2, 4)
    out, w, _, _ = oracle.attend(q, k, k, [[0]])
    assert not out.any() and not w.any()
    out, w, _, _ = oracle.attend(q, k, k, [[1]])          # one token, three queries: only the last sees it
    assert out[0, 0, 0, :, 0].tolist() == [0, 0, 1] and w[0, 0].tolist() == [1, 0]


@pytest.mark.parametrize("N,budget,recent", [(1, 1, 0), (9, 4, 2), (9, 4, 4), (9, 4, 0), (40, 17, 5), (40, 39, 1), (40, 40, 3)])
def test_evict_keeps_the_heaviest_and_the_last(N, budget, recent):
    g = torch.Generator().manual_seed(N * 100 + budget)
    w = torch.rand(6, N, generator=g)
    w[1] = torch.round(w[1] * 3)
    w[2] = 1.0
    if N > 4:
        w[3, 1::2] = float("nan")
        w[4, 0], w[4, 1], w[4, 2] = -0.0, 0.0, float("-inf")
    lens = [N, N, N, N, N, min(N, budget)]
    source, new = oracle.evict(w, lens, [budget] * 6, recent)
    for r in range(6):
        n = lens[r]
        if n <= budget:
            assert new[r] == n and source[r].tolist() == list(range(N))
            continue
        assert new[r] == budget
        got = source[r, :budget].tolist()
        assert got[budget - recent:] == list(range(n - recent, n))
        cand = range(n - recent)
        key = lambda i: (1, 0.0, i) if math.isnan(w[r, i]) else (0, -(float(w[r, i]) + 0.0), i)  # noqa: E731
        want = set(sorted(cand, key=key)[:budget - recent])
        assert set(got[:budget - recent]) == want
        moved = [(j, i) for j, i in enumerate(got[:budget - recent]) if i != j]
        assert all(i >= budget - recent for _, i in moved) and [i for _, i in moved] == sorted(i for _, i in moved)
        assert source[r, budget:].tolist() == list(range(budget, N))
