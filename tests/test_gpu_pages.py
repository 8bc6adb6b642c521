"""sfa_page_tables against the oracle's step-by-step page allocator: whole numbers,
so everything is equal."""
import numpy as np
import pytest
import torch

import oracle
import paper_2603_22300_amd as sfa

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)


def _state(rng, B, P, mp, num, most, spare):
    """Sequences that hold pages of a shuffled pool, and a free list of the rest."""
    old = rng.integers(0, most + 1, B)
    ids = rng.permutation(num)
    table, at = np.full((B, mp), -1), 0
    for b in range(B):
        h = -(-int(old[b]) // P)
        table[b, :h] = ids[at:at + h]
        at += h
    n = min(spare, num - at)
    free = np.full(num, -5)
    free[:n] = ids[at:at + n]
    return old, table, free, n


def _check(old, new, table, free, n, P, num, rows, old_null=False, alias=False):
    wt, wf = table.copy(), free.copy()
    got, left, starts, slots, pos = oracle.page_tables(old, new, wt, wf, n, P, num, rows)
    gt, gf, fin = _t(table), _t(free), _t([n])
    out = dict(slots=_t(np.full(rows, 77)), pos=_t(np.full(rows, 77))) if rows else {}
    for _ in range(1 if alias else 2):  # again with the same result, unless the count is updated in place
        g, left_t, s, sl, p = sfa.sfa_page_tables(None if old_null else _t(old), _t(new), gt, gf, fin, P,
                                                  free_out=fin if alias else None, **out)
        torch.cuda.synchronize()
        for x, y in ((gt, wt), (gf, wf), (g, got), (s, starts)) + (((sl, slots), (p, pos)) if rows else ()):
            assert np.array_equal(x.cpu().numpy(), y)
        assert int(left_t) == left
    return got, left


@pytest.mark.parametrize("B,P,mp,num,most,spare,rows", [
    (1, 16, 4, 8, 64, 8, 100),
    (64, 16, 20, 700, 300, 200, 4000),          # one launch
    (64, 16, 20, 700, 300, 30, 9000),           # two launches, pages run out
    (1500, 1, 3, 3000, 3, 500, 2000),           # more sequences than threads, single-position pages
    (5000, 8, 4, 20000, 32, 4000, 60000),
    (3, 128, 40, 130, 5000, 100, 12345),
    (7, 2, 9, 60, 18, 5, 0),                    # tables only
])
@pytest.mark.parametrize("alias", [False, True])
def test_page_tables(B, P, mp, num, most, spare, rows, alias):
    rng = np.random.default_rng(B + P)
    old, table, free, n = _state(rng, B, P, mp, num, most, spare)
    r = rng.random(B)
    new = np.where(r < 0.3, old + 1, np.where(r < 0.5, 0, np.where(r < 0.6, old // 2, rng.integers(0, mp * P + 1, B))))
    _check(old, new, table, free, n, P, num, rows, alias=alias)


def test_lengths_outside_the_capacity_and_from_nothing():
    table, free = np.full((4, 3), -1), np.arange(12)
    _check([0, 0, 0, 0], [-3, 100, 13, 24], table, free, 12, 8, 12, 70, old_null=True)
    table[1] = [4, 5, 6]
    _check([-1, 50, 0, 0], [5, 24, 0, -9], table, free, 3, 8, 12, 40)
    _check([0, 0, 0, 0], [5, 24, 0, 1], np.full((4, 3), -1), free, -4, 8, 12, 40)      # no free page at all
    _check([0, 0, 0, 0], [5, 24, 0, 1], np.full((4, 3), -1), free, 99, 8, 12, 40)      # a count past the list


def test_pages_given_back_are_taken_in_the_same_call():
    table = np.array([[0, 1, 2], [-1, -1, -1]])
    got, left = _check([12, 0], [2, 9], table, np.zeros(3), 0, 4, 3, 9)
    assert got.tolist() == [2, 8] and left == 0


def test_bad_page_ids_get_no_slot():
    table = np.array([[9, -1], [1, 0]])
    free = np.array([7, 2, 0])
    _check([3, 5], [8, 8], table, free, 2, 4, 3, 12)


def test_more_tokens_than_an_int_holds():
    """2^20 sequences from nothing to 2^13 positions each: 2^33 tokens asked for, none got
    (no page is free); the rows' starts stop at 2^31 - 1."""
    B = 1 << 20
    new = torch.full((B,), 1 << 13, dtype=torch.int32, device=DEV)
    z = torch.zeros((1,), dtype=torch.int32, device=DEV)
    got, left, starts, slots, pos = sfa.sfa_page_tables(None, new, torch.zeros((B, 1), dtype=torch.int32, device=DEV),
                                                        torch.zeros((4,), dtype=torch.int32, device=DEV), z, 1 << 13,
                                                        n_rows=10000)
    torch.cuda.synchronize()
    assert int(got.abs().sum()) == 0 and int(left) == 0 and bool((slots == -1).all())
    want = np.minimum(np.arange(B + 1, dtype=np.int64) << 13, 2 ** 31 - 1)
    assert np.array_equal(starts.cpu().numpy(), want)
    assert np.array_equal(pos.cpu().numpy(), np.arange(10000) % (1 << 13))


def test_page_tables_refusals():
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    with pytest.raises(ValueError):
        sfa.sfa_page_tables(i(3), i(4), i(4, 2), i(8), i(1), 16)
    with pytest.raises(ValueError):
        sfa.sfa_page_tables(i(4), i(4), i(3, 2), i(8), i(1), 16)
    with pytest.raises(TypeError):
        sfa.sfa_page_tables(i(4), i(4), i(4, 2), i(8), i(1).long(), 16)
    with pytest.raises(sfa.SfaError):
        sfa.sfa_page_tables(i(4), i(4), i(4, 2), i(8), i(1), 12)
    with pytest.raises(sfa.SfaError) as e:
        sfa.sfa_page_tables(i(4), i(4), i(4, 2), i(8), i(1), 16, ws=i(1))
    assert e.value.status == sfa.SFA_ENOSPC
    x = i(4)
    with pytest.raises(sfa.SfaError):
        sfa.sfa_page_tables(x, i(4), i(4, 2), i(8), i(1), 16, got=x)
