"""Pins of the oracle's step tables, chunk attention and logit adjustment: vectors
worked by hand, a replay with sets of pages, and torch's attention with a mask."""
import math

import numpy as np
import pytest
import torch

from oracle import kap_oracle as O


def test_tables_worked():
    # 20 tokens on pages 5, 6 lose 3 (17 kept), and get 4: 21 on two pages still
    # 16 on page 7 get one: a second page, the first free one
    # 40 on pages 1, 2, 3 end: they go back in order
    # nothing, then 33 tokens: three pages
    table = [[5, 6, -1], [7, -1, -1], [1, 2, 3], [-1, -1, -1]]
    ring = [-1, 8, 9, 10, 11, -1, -1, -1]                          # 8 9 10 11 from entry 1 on
    got = O.step_tables([20, 16, 40, 0], [4, 1, 0, 33], table, ring, (1, 4), 40,
                        keep=[17, 16, 0, 0])
    assert got["block_table"].tolist() == [[5, 6, -1], [7, 8, -1], [1, 2, 3], [9, 10, 11]]
    assert got["free_pages"].tolist() == [-1, 8, 9, 10, 11, 1, 2, 3]
    assert got["free_out"].tolist() == [5, 3]
    assert got["new_lens"].tolist() == [21, 17, 0, 33] and got["status"].tolist() == [0] * 4
    assert got["q_offsets"].tolist() == [0, 4, 5, 5, 38]
    assert got["slot_mapping"].tolist() == [6 * 16 + 1, 6 * 16 + 2, 6 * 16 + 3, 6 * 16 + 4, 8 * 16,
                                            *range(9 * 16, 12 * 16 - 15), -1, -1]
    assert got["positions"].tolist() == [17, 18, 19, 20, 16, *range(33), 0, 0]


def test_tables_refusals():
    lens, add = [5, 5, 5, -1, 5, 31, 16, 3, 16], [1, -1, 1, 1, 28, 3, 1, 9, 1]
    keep = [5, 5, 6, 0, 5, 31, 16, 3, 16]
    table = np.arange(18).reshape(9, 2)
    got = O.step_tables(lens, add, table, [90, 91], (0, 1), 12, keep=keep)
    #   ok, add < 0, keep > len, len < 0, 33 tokens > 2 pages, 34 > 2 pages, takes the one page,
    #   11 tokens, 12 tokens and no page left
    assert got["status"].tolist() == [0, 1, 1, 1, 2, 2, 0, 0, 4]
    assert got["new_lens"].tolist() == [6, 5, 5, -1, 5, 31, 17, 12, 16]
    assert got["q_offsets"].tolist() == [0, 1, 1, 1, 1, 1, 1, 2, 11, 11]
    assert got["free_out"].tolist() == [1, 0]
    got = O.step_tables(lens, add, table, [90, 91], (0, 2), 10, keep=keep)
    assert got["status"].tolist() == [0, 1, 1, 1, 2, 2, 0, 3, 3]
    # what a refused sequence no longer keeps goes back all the same; pinned pages stay
    got = O.step_tables([32, 32], [33, 0], [[1, 2], [3, 4]], [0] * 4, (2, 0), 50, keep=[0, 0],
                        pinned=[0, 1])
    assert got["status"].tolist() == [2, 0] and got["new_lens"].tolist() == [0, 0]
    assert got["free_pages"].tolist() == [4, 0, 1, 2] and got["free_out"].tolist() == [2, 3]


def test_tables_keep_every_page_once():
    # pages move between rows and the ring; none is lost or held twice
    rng = np.random.default_rng(3)
    B, stride, pages = 7, 12, 40
    lens, table = np.zeros(B, np.int64), np.full((B, stride), -1)
    ring, state = rng.permutation(pages), (0, pages)
    for _ in range(200):
        keep = [int(rng.integers(0, L + 1)) if rng.random() < 0.4 else int(L) for L in lens]
        add = rng.integers(0, 70, B)
        got = O.step_tables(lens, add, table, ring, state, 150, keep=keep)
        lens, table, ring, state = (got[k] for k in ("new_lens", "block_table", "free_pages",
                                                     "free_out"))
        held = [table[b, j] for b in range(B) for j in range(-(-lens[b] // 16))]
        free = [ring[(state[0] + i) % pages] for i in range(state[1])]
        assert sorted(held + free) == list(range(pages))
        assert (got["slot_mapping"][:got["q_offsets"][-1]] >= 0).all()


@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 0), (5, 0), (5, 3), (40, 2), (1, 100)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_chunks_against_torch(dtype, window, sinks):
    rng = np.random.default_rng(window + sinks)
    Hq, Hkv, D, P = 4, 2, 16, 9
    new, lens = [1, 7, 0, 20], [33, 40, 5, 20]
    table = np.stack([rng.permutation(P)[:3] for _ in lens])
    table[1, 1] = table[0, 0]
    if dtype == "f32":
        k, v = (rng.standard_normal(s).astype(np.float32) for s in ((P, Hkv, D // 8, 16, 8),
                                                                    (P, Hkv, D, 16)))
        sc = None
    elif dtype == "bf16":
        k, v = (torch.randn(s).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
                for s in ((P, Hkv, D // 8, 16, 8), (P, Hkv, D, 16)))
        sc = None
    else:
        k, v = (rng.integers(0, 120, s).astype(np.uint8) for s in ((P, Hkv, D // 8, 16, 8),
                                                                    (P, Hkv, D, 16)))
        sc = rng.uniform(0.001, 0.01, (P, 2)).astype(np.float32)
    pool = O.KVPool(k, v, dtype, sc)
    offs = np.concatenate([[0], np.cumsum(new)])
    q = rng.standard_normal((offs[-1] + 2, Hq, D))
    o, lse = O.chunk_attention(pool, q, offs, lens, table, 0.3, window, sinks)
    assert not o[-2:].any()
    for b, (n, L) in enumerate(zip(new, lens)):
        if n == 0:
            continue
        t, p = torch.arange(L), torch.arange(L - n, L)[:, None]
        mask = t <= p
        if window:
            mask &= (t > p - window) | (t < sinks)
        for h in range(Hq):
            kk = np.concatenate([pool.keys(np.array([x]), h // 2)[0] for x in table[b]])[:L]
            vv = np.concatenate([pool.values(np.array([x]), h // 2)[0] for x in table[b]])[:L]
            qq = torch.as_tensor(q[offs[b]:offs[b + 1], h])
            z = (qq @ torch.as_tensor(kk).T * 0.3).masked_fill(~mask, -math.inf)
            assert np.allclose(torch.logsumexp(z, 1), lse[offs[b]:offs[b + 1], h], atol=1e-10)
            assert np.allclose(z.softmax(1) @ torch.as_tensor(vv), o[offs[b]:offs[b + 1], h],
                               atol=1e-10)


def test_chunks_of_verify_and_of_more_rows_than_tokens():
    rng = np.random.default_rng(2)
    pool = O.KVPool(rng.standard_normal((6, 1, 2, 16, 8)).astype(np.float32),
                    rng.standard_normal((6, 1, 16, 16)).astype(np.float32), "f32", None)
    table, lens = np.array([[0, 1, 2], [3, 4, 9]]), [40, 3]
    q = rng.standard_normal((2, 5, 2, 16))
    o, lse = O.verify(pool, q, lens, table, 0.2)
    oc, lc = O.chunk_attention(pool, q.reshape(10, 2, 16), [0, 5, 10], lens, table, 0.2)
    assert np.array_equal(o.reshape(10, 2, 16), oc) and np.array_equal(lse.reshape(10, 2), lc)
    assert np.isneginf(lc[5:7]).all() and not oc[5:7].any()       # before the first token


def test_logits_worked():
    x = [2.0, -2.0, 0.0, 4.0, 1.0, -math.inf, 3.0]
    got = O.adjust_logits(x, prompt=[0, 1, 99], told=[3, 0, 3, -1, 5], repetition=2.0,
                          frequency=0.25, presence=0.5, biases=[(4, 1.0), (6, 9.0), (6, -1.0), (7, 1)],
                          allowed=[1, 1, 0, 1, 1, 1, 1])
    # 0: 2 / 2 - 0.25 - 0.5; 1: -2 * 2; 3: 4 / 2 - 0.5 - 0.5; 4: 1 + 1; 6: 3 - 1
    assert got.tolist() == [0.25, -4.0, -math.inf, 1.0, 2.0, -math.inf, 2.0]
    assert O.adjust_logits(x).tolist() == x
