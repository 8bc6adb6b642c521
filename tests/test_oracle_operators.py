"""Pins of the oracle of rotary positions, page tables and the 4-bit cache: closed
forms, invariants and hand-worked cases (no GPU)."""
import math

import numpy as np
import pytest

import oracle
import paper_2603_22300_amd as sfa


@pytest.mark.parametrize("sections,order", [([8], "sections"), ([2, 3, 3], "sections"),
                                            ([2, 3, 3], "interleaved"), ([4, 1], "own"), ([1, 5, 2], "interleaved")])
def test_ladder_is_the_plan(sections, order):
    # libsfa's plan (host code) against the definition
    axis, freq = oracle.rope_ladder(sections, 5e5, order)
    plan = sfa.sfa_rope_plan(2 * sum(sections) + 4, sections, theta=5e5, order=order)
    assert plan.rot == 2 * sum(sections) and plan.naxes == len(sections)
    assert plan.axis == axis.tolist()
    assert np.allclose(plan.freq, freq, rtol=1e-15, atol=0)
    assert [plan.axis.count(a) for a in range(len(sections))] == sections
    if order != "own":
        assert plan.freq == sorted(plan.freq, reverse=True) and plan.freq[0] == 1.0


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_rope_turns_pairs(pairing):
    rng = np.random.default_rng(1)
    axis, freq = oracle.rope_ladder([2, 1], 100.0, "sections")
    x = rng.standard_normal((2, 3, 5, 8))
    pos = rng.integers(-50, 50, (2, 2, 5))
    y = oracle.rope(x, pos, axis, freq, pairing)
    assert np.array_equal(y[..., 6:], x[..., 6:])                       # past rot: copied
    u, v = oracle.rope_pairs(6, pairing)
    z = (x[..., u] + 1j * x[..., v]) * np.exp(1j * np.stack([pos[a][:, None] * f for a, f in zip(axis, freq)], -1))
    assert np.allclose(y[..., u], z.real, atol=1e-14) and np.allclose(y[..., v], z.imag, atol=1e-14)
    assert np.allclose(oracle.rope(y, pos, axis, freq, pairing, inverse=True), x, atol=1e-13)
    # a score depends on the difference of positions only
    q, k = x[:1, :1, :1], x[1:, 1:2, 1:2]
    dot = lambda p, r: float((oracle.rope(q, np.full((2, 1, 1), p), axis, freq, pairing)  # noqa: E731
                              * oracle.rope(k, np.full((2, 1, 1), r), axis, freq, pairing)).sum())
    assert math.isclose(dot(7, 3), dot(104, 100), rel_tol=1e-12)


def test_page_tables_by_hand():
    # pages of 4; sequence 0 grows 3 -> 6 (one page), 1 ends (two pages back), 2 starts with 9 (three pages)
    table = np.array([[5, -1, -1], [7, 8, -1], [-1, -1, -1]])
    free = np.array([1, 2, 0, 0, 0, 0, 0, 0, 0])
    got, n, starts, slots, pos = oracle.page_tables([3, 8, 0], [6, 0, 9], table, free, 2, 4, 9, 14)
    assert table.tolist() == [[5, 8, -1], [7, 8, -1], [7, 2, 1]]
    assert (got.tolist(), n, starts.tolist()) == ([6, 0, 9], 0, [0, 3, 3, 12])
    assert pos.tolist() == [3, 4, 5] + list(range(9)) + [-1, -1]
    assert slots.tolist() == [23, 32, 33] + [28, 29, 30, 31, 8, 9, 10, 11, 4] + [-1, -1]
    # too few pages: the last sequence stops where they end
    table = np.full((2, 3), -1)
    got, n, starts, slots, pos = oracle.page_tables([0, 0], [5, 9], table, np.array([3, 1, 0]), 3, 4, 4, 20)
    assert got.tolist() == [5, 4] and n == 0 and (slots >= 0).sum() == 9


def test_page_tables_conserve_pages():
    rng = np.random.default_rng(2)
    B, mp, P, num = 6, 5, 8, 20
    table, free, n = np.full((B, mp), -1), np.arange(num), num
    lens = np.zeros(B, int)
    for _ in range(60):
        new = rng.integers(0, mp * P + 1, B)
        got, n, _, _, _ = oracle.page_tables(lens, new, table, free, n, P, num, 0)
        assert (got <= new).all()
        lens = np.where(new > lens, got, new)
        held = [int(table[b, j]) for b in range(B) for j in range(-(-lens[b] // P))]
        # a sequence that found too few pages holds those it found
        assert sorted(held + free[:n].tolist()) == list(range(num))


def test_quant_q4_rows():
    q, s = oracle.quant_q4(np.array([[7.0, -7.0, 0.5, 1.5, 2.5, -0.5, -1.5, 3.0], [0.0] * 8], np.float32))
    assert s.tolist() == [1.0, 0.0]
    assert q.tolist() == [[7, -7, 0, 2, 2, 0, -2, 3], [0] * 8]
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((3000, 32)) * np.exp(rng.uniform(-20, 20, (3000, 1)))).astype(np.float32)
    for bf in (False, True):
        q, s = oracle.quant_q4(x, bf)
        assert np.abs(q).max() == 7
        # half a step, and 7 (2^-8) steps where the bfloat16 scale came out below max / 7
        assert (np.abs(x - q * s.astype(np.float64)[:, None]) <= s[:, None] * (0.5 + (7 * 2.0 ** -8 if bf else 1e-6))).all()
    assert np.array_equal(oracle.unpack_q4(oracle.pack_q4(q)), q)
    assert oracle.pack_q4(np.array([-7, 3])).tolist() == [0x39]
