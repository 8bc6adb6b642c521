"""GPU parity of the 4-bit cache: sfa_kv_append_q4 bit for bit against the oracle's
coding and quantisation, sfa_attn_decode_q4 against the oracle's decode of the values
the cache stands for."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2603_22300_amd as sfa
import sfa_inputs as si
from helpers import np_f64, oracle_topk_rows

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _cache(pages, Hkv, P, d, k):
    rows = (pages, Hkv, P)
    return [torch.full(rows + (k,), 201, dtype=torch.uint8, device=DEV),
            torch.full(rows + (k // 2,), 202, dtype=torch.uint8, device=DEV),
            torch.full(rows, -1.0, device=DEV),
            torch.full(rows + (d // 2,), 203, dtype=torch.uint8, device=DEV),
            torch.full(rows + (d // 32,), -2.0, dtype=torch.bfloat16, device=DEV)]


def _kv(B, Hkv, T, d, seed, kt, vt):
    """Keys and values with rows of unlike size: zeros, subnormals and large ones among them."""
    k = si.normal((B, Hkv, T, d), seed, "k", device=DEV)
    v = si.normal((B, Hkv, T, d), seed, "v", device=DEV)
    flat = v.view(-1, d)
    for i, f in enumerate((0.0, 1e-42, 1e-30, 1e20, 3e36)):
        if flat.shape[0] > 2 * i:
            flat[2 * i, :32] *= f
            k.view(-1, d)[2 * i] *= f
    return k.to(kt), v.to(vt)


def _expect(cache, k_new, v_new, k, where):
    """The oracle's cache after writing token (b, t) to where[b, t] = (page, slot) or None."""
    want = [c.float().cpu().numpy() if c.dtype == torch.bfloat16 else c.cpu().numpy().copy() for c in cache]
    kk, vv = k_new.float().cpu().numpy(), v_new.float().cpu().numpy()
    new = oracle.rows_q4(kk, vv, k)
    B, Hkv, T, _ = kk.shape
    for b in range(B):
        for t in range(T):
            if where[b][t] is None:
                continue
            page, slot = where[b][t]
            for w, x in zip(want, new):
                w[page, :, slot] = x[b, :, t]
    return want, new


def _same(cache, want):
    for c, w in zip(cache, want):
        got = c.float().cpu().numpy() if c.dtype == torch.bfloat16 else c.cpu().numpy()
        assert np.array_equal(got, w)


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("B,Hkv,T,P,d,k,kt,vt", [
    (2, 2, 37, 16, 128, 16, F32, BF16),
    (1, 1, 1, 64, 64, 8, BF16, F32),
    (3, 5, 9, 32, 96, 24, BF16, BF16),
    (1, 3, 20, 16, 256, 32, F32, F32),
    (2, 1, 12, 16, 32, 32, F32, BF16),       # every coordinate kept
    (1, 2, 6, 128, 224, 120, F32, F32),
])
@pytest.mark.parametrize("packed", [False, True])
def test_append_through_slots(B, Hkv, T, P, d, k, kt, vt, packed):
    kn, vn = _kv(B, Hkv, T, d, d + k, kt, vt)
    if packed:  # [tokens, heads, d] buffers, k and v views of one projection
        both = torch.cat((kn, vn.to(kt)), 1).transpose(1, 2).contiguous()
        kn, vn = both[:, :, :Hkv].transpose(1, 2), both[:, :, Hkv:].transpose(1, 2)
    pages = -(-T // P) * B + 3
    rng = np.random.default_rng(T)
    slots = rng.permutation(pages * P)[:B * T].reshape(B, T)
    slots[rng.random((B, T)) < 0.15] = -1
    slots[0, 0] = pages * P if T > 1 else slots[0, 0]    # outside the pool
    where = [[divmod(int(s), P) if 0 <= s < pages * P else None for s in row] for row in slots]
    cache = _cache(pages, Hkv, P, d, k)
    want, new = _expect(cache, kn, vn, k, where)
    out = dict(k_idx=torch.full((B, Hkv, T, k), -3, dtype=torch.int16, device=DEV),
               k_val=torch.full((B, Hkv, T, k), -3.0, device=DEV),
               v_out=torch.full((B, Hkv, T, d), -3.0, dtype=BF16, device=DEV))
    st = torch.from_numpy(slots.astype(np.int32)).to(DEV)
    sfa.sfa_kv_append_q4(kn, vn, None, *cache, k=k, slots=st, **out)
    torch.cuda.synchronize()
    _same(cache, want)
    kv, v = oracle.values_q4(new[1], new[2], new[3], new[4])
    skip = np.array([[w is None for w in row] for row in where])[:, None, :, None]
    for name, x in (("k_idx", new[0]), ("k_val", kv.astype(np.float32)),
                    ("v_out", torch.from_numpy(v).to(BF16).float().numpy())):
        assert np.array_equal(out[name].float().cpu().numpy(), np.where(skip, -3, x).astype(np.float32)), name
    # without the extra outputs, and over a contiguous cache's slots: the same rows
    again = _cache(pages, Hkv, P, d, k)
    sfa.sfa_kv_append_q4(kn, vn, None, *again, k=k, slots=st)
    _same(again, want)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("B,Hkv,T,d,k", [(5, 2, 1, 128, 16), (5, 8, 3, 64, 8), (5, 3, 40, 96, 8)])
def test_append_by_lengths(B, Hkv, T, d, k, paged):
    """A sequence in its first page, one across a page's end, a full one, one with nothing
    to append, one whose page lies outside the pool; lengths clamped and advanced."""
    P, mp = 16, 4
    cap = P * mp
    lens, n_new = [3, 15, cap, 7, -2], [T, T + 5, T, 0, T]
    kn, vn = _kv(B, Hkv, T, d, T, F32, BF16)
    table = np.random.default_rng(T).permutation(B * mp).reshape(B, mp)
    if paged:
        table[4, 0] = B * mp + 2
    cache = _cache(B * mp, Hkv, P, d, k) if paged else _cache(B, Hkv, cap, d, k)
    where = [[None] * T for _ in range(B)]
    for b in range(B):
        for t in range(min(n_new[b], T)):
            pos = max(lens[b], 0) + t
            if pos >= cap:
                continue
            page, slot = (int(table[b, pos // P]), pos % P) if paged else (b, pos)
            if page < B * mp:
                where[b][t] = (page, slot)
    want, _ = _expect(cache, kn, vn, k, where)
    L = torch.tensor(lens, dtype=torch.int32, device=DEV)
    sfa.sfa_kv_append_q4(kn, vn, L, *cache, k=k, n_new=torch.tensor(n_new, dtype=torch.int32, device=DEV),
                         block_table=torch.from_numpy(table.astype(np.int32)).to(DEV) if paged else None)
    torch.cuda.synchronize()
    _same(cache, want)
    assert L.tolist() == [min(cap, max(0, a) + min(n, T)) for a, n in zip(lens, n_new)]
    empty = kn[:, :, :0]
    sfa.sfa_kv_append_q4(empty, vn[:, :, :0], L, *cache, k=k,
                         block_table=torch.from_numpy(table.astype(np.int32)).to(DEV) if paged else None)
    _same(cache, want)


def _filled(B, Hkv, L, d, k, P, seed, vmul=None):
    """A cache filled by sfa_kv_append_q4 (contiguous, or pages of P in random order) and the
    values it stands for as the oracle has them."""
    kn = si.normal((B, Hkv, L, d), seed, "k", device=DEV)
    vn = si.normal((B, Hkv, L, d), seed, "v", device=DEV)
    if vmul is not None:
        vn = vn * vmul
    table = None
    if P:
        mp = -(-L // P)
        g = torch.Generator().manual_seed(seed)
        table = torch.randperm(B * mp + 2, generator=g)[:B * mp].reshape(B, mp).to(torch.int32).to(DEV)
        cache = _cache(B * mp + 2, Hkv, P, d, k)
    else:
        cache = _cache(B, Hkv, L, d, k)
    sfa.sfa_kv_append_q4(kn, vn, torch.zeros(B, dtype=torch.int32, device=DEV), *cache, k=k, block_table=table)
    ci, cv = oracle_topk_rows(kn.cpu().numpy().reshape(-1, d), k)
    kq, ks = oracle.quant_q4(cv)
    vq, vs = oracle.quant_q4(vn.cpu().numpy().reshape(B * Hkv * L, -1, 32), bf16_scale=True)
    kv = kq.astype(np.float64) * ks.astype(np.float64)[:, None]
    vv = (vq.astype(np.float64) * vs.astype(np.float64)[..., None]).reshape(B, Hkv, L, d)
    return cache, table, ci.reshape(B, Hkv, L, k), kv.reshape(B, Hkv, L, k), vv


def _bounds(qv, kv, vv, scale, k, L):
    """Derived bounds on O (absolute, per KV head's largest |v|) and LSE.
    A base-2 exponent t = scale log2(e) ks sum of k products is off by at most (k + 4)
    2^-24 times A = |scale| log2(e) k max|q| max|k| (a bound on the sum of its
    magnitudes), v_exp_f32 by 2^-22 relative, and a weight's rounding to a whole number by
    2^-28 of the largest weight, which is more of a small one: taken as 2^-22 relative,
    so a weight is off by w = ln 2 * dt + 2^-21 relative; O's numerator and denominator each
    carry that, and sums of n terms in float32 another (trees and chains of at most 64
    merges) 128 * 2^-24."""
    A = abs(scale) * 1.4427 * k * np.abs(qv).max() * np.abs(kv).max()
    w = math.log(2) * (k + 4) * 2.0 ** -24 * A + 2.0 ** -21
    return (2 * w + 256 * 2.0 ** -24), w + 64 * 2.0 ** -24


def _decode(B, Hkv, G, L, d, k, P, seq, window=0, n_global=0, dense=False, seed=0, scale=None, vmul=None,
            o_dtype=torch.float32, qmul=1.0):
    seed = seed or (L + d + k)
    cache, table, ci, kv, vv = _filled(B, Hkv, L, d, k, P, seed, vmul)
    Hq = Hkv * G
    q = si.normal((B, Hq, d), seed, "q", device=DEV) * qmul
    qi, qv = sfa.sfa_topk_encode(q, k)
    scale = scale or 1.0 / math.sqrt(d)
    kw = dict(q=q) if dense else dict(q_idx=qi, q_val=qv)
    sl = torch.tensor(seq, dtype=torch.int32, device=DEV) if seq is not None else None
    o, lse = sfa.sfa_attn_decode_q4(*cache, block_table=table, seq_len=sl, scale=scale, window=window,
                                    n_global=n_global, o_dtype=o_dtype, **kw)
    torch.cuda.synchronize()
    lens = [min(max(s, 0), P * -(-L // P) if P else L) for s in (seq or [L] * B)]
    oqi, oqv = qi.cpu().numpy(), qv.cpu().numpy()
    tol_o, tol_l = _bounds(oqv, kv, vv, scale, k, L)
    for b in range(B):
        if lens[b] == 0:
            assert not o[b].any() and bool((lse[b] == -math.inf).all())
            continue
        O, E = oracle.attn_decode(oqi[b:b + 1], oqv[b:b + 1], ci[b:b + 1], kv[b:b + 1], vv[b:b + 1], d, scale,
                                  seq_len=[lens[b]], window=window, n_global=n_global)
        # per run of 32 coordinates: each has its own scales
        vmax = np.abs(vv[b, :, :lens[b]]).reshape(Hkv, -1, d // 32, 32).max((1, 3))
        bound = tol_o * np.repeat(np.repeat(vmax, 32, -1), G, 0) + 1e-44
        if o_dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * np.abs(O[0])
        err = np.abs(np_f64(o[b]) - O[0])
        assert (err <= bound).all(), (b, float((err / bound).max()))
        assert np.abs(np_f64(lse[b]) - E[0]).max() <= tol_l + 2.0 ** -23 * np.abs(E).max()
    return o, lse


@pytest.mark.parametrize("B,Hkv,G,L,d,k,P,seq", [
    (3, 2, 4, 300, 128, 16, 0, [300, 1, 157]),
    (4, 1, 8, 4097, 128, 16, 64, [4097, 2049, 0, 64]),
    (2, 2, 1, 777, 64, 16, 0, None),
    (2, 1, 3, 1000, 64, 8, 16, [999, 17]),
    (2, 2, 6, 500, 96, 24, 32, [500, 33]),
    (1, 1, 5, 70, 32, 32, 16, [65]),
    (2, 1, 4, 260, 256, 16, 256, [257, 100]),
    (1, 2, 7, 150, 224, 40, 0, [150]),
    (3, 1, 2, 1, 128, 8, 0, [1, 0, 1]),
    (2, 1, 4, 90, 160, 160, 16, [90, 64]),       # every coordinate kept
    (5, 3, 4, 2000, 128, 32, 128, [2000, 5000, -4, 1999, 1]),
])
def test_decode_q4(B, Hkv, G, L, d, k, P, seq):
    if seq is not None and P == 0:
        seq = [min(s, L) for s in seq]
    # lengths past the tokens appended read pages of no tokens: keep those that were written
    if seq is not None:
        seq = [min(s, L) for s in seq]
    _decode(B, Hkv, G, L, d, k, P, seq)
    _decode(B, Hkv, G, L, d, k, P, seq, dense=True, o_dtype=torch.bfloat16)


def test_decode_q4_window():
    _decode(2, 2, 4, 5000, 128, 16, 64, [5000, 3000], window=1000, n_global=3, dense=True)
    _decode(2, 1, 2, 700, 64, 8, 0, [700, 90], window=1, n_global=0)       # the last key alone
    _decode(3, 1, 4, 3000, 128, 16, 16, [2900, 2, 500], window=100, n_global=400)


@pytest.mark.parametrize("P", [0, 16, 64])
@pytest.mark.parametrize("k", [8, 16, 24, 32])
@pytest.mark.parametrize("G", [3, 8])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 192, 256])
def test_decode_q4_forms(d, G, k, P):
    """Every head dimension, group, code count and paging has a kernel of its own: whole
    blocks of keys, a last one of one key or some, and a sequence of one key."""
    _decode(3, 1, G, 387, d, k, P, [387, 321, 1], dense=G == 3)


@pytest.mark.parametrize("d,G,L", [(64, 4, 64), (64, 8, 50), (128, 4, 64), (128, 2, 200), (96, 3, 33), (256, 8, 64),
                                   (64, 4, 4096), (128, 8, 4000)])
def test_decode_q4_products_keep_float32_accuracy(d, G, L):
    """Weights of very different sizes times the cached numbers, element by element
    against the sum of the magnitudes of its terms, S = sum p |v|.  Queries of one
    coordinate, so that a base-2 exponent is one product and off by at most 5 * 2^-24 times
    A, the largest of them (the key's scale, the query, the score's scale, the difference
    with the maximum), and a weight by w = ln 2 * that + 2^-22 (v_exp_f32) relative; the
    output carries a weight's error twice (numerator and sum), and at most 20 roundings of
    2^-24 in sums and joins; a weight's rounding to a whole number is 2^-28 of the largest
    p times the largest scale, 7 of which are at most max |v|.  Over many keys the
    errors of single weights are as unlike as the numbers they multiply: both the output and
    its error grow as the root of their number, and the 2-norms are in a ratio of w at most;
    2 w is asked for."""
    k, Hkv, B, seed = 16, 2, 2, 77
    cache, _, ci, kv, vv = _filled(B, Hkv, L, d, k, 0, seed, None)
    q = si.normal((B, Hkv * G, d), seed, "q", device=DEV)
    qi, qv = sfa.sfa_topk_encode(q, k)
    qv[..., 0], qv[..., 1:] = 3.0, 0.0
    scale = 1.0
    o, _ = sfa.sfa_attn_decode_q4(*cache, q_idx=qi, q_val=qv, o_dtype=torch.float32, scale=scale)
    for b in range(B):
        args = [x.cpu().numpy()[b:b + 1] for x in (qi, qv)] + [ci[b:b + 1], kv[b:b + 1]]
        O, _ = oracle.attn_decode(*args, vv[b:b + 1], d, scale)
        S, _ = oracle.attn_decode(*args, np.abs(vv[b:b + 1]), d, scale)
        A = 1.4427 * scale * 3.0 * 2 * np.abs(kv[b]).max()
        w = math.log(2) * 5 * 2.0 ** -24 * A + 2.0 ** -22
        vmax = np.abs(vv[b]).reshape(Hkv, -1, d // 32, 32).max((1, 3))
        bound = (2 * w + 20 * 2.0 ** -24) * S[0] + 2.0 ** -28 * L / 7 * np.repeat(np.repeat(vmax, 32, -1), G, 0)
        err = np.abs(np_f64(o[b]) - O[0])
        assert (err <= bound).all(), (b, float((err / bound).max()))
        ratio = np.linalg.norm(err) / np.linalg.norm(O)
        assert L < 1000 or ratio <= 2 * w, (b, ratio, w)


def test_decode_q4_scales_of_any_size():
    """Runs of a value row, and rows, of magnitudes from 2^-120 to 2^120: the weights keep
    float32 accuracy of each run.  Large scores and both signs of the scale."""
    mul = torch.ones((1, 1, 200, 128), device=DEV)
    mul[..., :32] = 2.0 ** 100
    mul[..., 32:64] = 1e4
    mul[..., 64:96] = 2.0 ** 90
    _decode(1, 1, 4, 200, 128, 16, 0, [200], vmul=mul * 2.0 ** -80)
    for m in (2.0 ** 120, 2.0 ** -100, 7e4, 1e-5):
        _decode(1, 2, 8, 150, 64, 16, 16, [150], vmul=m)
    grow = (2.0 ** torch.linspace(-60, 60, 300, device=DEV)).reshape(1, 1, 300, 1)
    _decode(1, 1, 4, 300, 128, 16, 0, [300], vmul=grow)
    _decode(1, 1, 4, 300, 128, 16, 0, [300], vmul=grow.flip(2))
    _decode(2, 1, 4, 900, 128, 16, 64, [900, 3], qmul=20.0)
    _decode(2, 1, 4, 900, 128, 16, 64, [900, 3], scale=-2.0, qmul=3.0)


def test_decode_q4_infinite_scales():
    """An infinite or NaN scale of a value run reaches its coordinates of the keys that are
    seen, and no others; of a key that is not seen, nothing.  A code scale that is NaN
    makes the head's output NaN."""
    B, Hkv, L, d, k, G = 2, 1, 200, 128, 16, 4
    cache, _, _, _, _ = _filled(B, Hkv, L, d, k, 0, 11, None)
    q = si.normal((B, G, d), 11, "q", device=DEV)
    lens = torch.tensor([150, 199], dtype=torch.int32, device=DEV)
    want = sfa.sfa_attn_decode_q4(*cache, seq_len=lens, q=q, o_dtype=torch.float32)
    bad = [x.clone() for x in cache]
    bad[4][0, 0, 150:] = float("inf")   # behind the sequence
    bad[2][0, 0, 150:] = float("nan")
    bad[4][1, 0, 70, 1] = float("inf")
    bad[4][1, 0, 3, 3] = float("nan")
    o, lse = sfa.sfa_attn_decode_q4(*bad, seq_len=lens, q=q, o_dtype=torch.float32)
    assert torch.equal(o[0], want[0][0]) and torch.equal(lse, want[1])
    nan = o[1].isnan().view(G, 4, 32)
    assert bool(nan[:, 1].all() and nan[:, 3].all()) and not bool(nan[:, 0].any() or nan[:, 2].any())
    assert torch.equal(o[1].view(G, 4, 32)[:, ::2], want[0][1].view(G, 4, 32)[:, ::2])
    bad[2][1, 0, 9] = float("nan")
    o, lse = sfa.sfa_attn_decode_q4(*bad, seq_len=lens, q=q, o_dtype=torch.float32)
    assert bool(o[1].isnan().all() and lse[1].isnan().all()) and torch.equal(o[0], want[0][0])


def test_decode_q4_is_the_same_paged_and_contiguous_and_repeatable():
    B, Hkv, L, d, k = 3, 2, 1500, 128, 16
    kn, vn = _kv(B, Hkv, L, d, 3, F32, BF16)
    vn = vn.float().clamp(-4, 4).to(BF16)
    kn = kn.clamp(-4, 4)
    q = si.normal((B, 8, d), 4, "q", device=DEV)
    flat = _cache(B, Hkv, L, d, k)
    sfa.sfa_kv_append_q4(kn, vn, torch.zeros(B, dtype=torch.int32, device=DEV), *flat, k=k)
    lens = torch.tensor([1500, 700, 1], dtype=torch.int32, device=DEV)
    o, lse = sfa.sfa_attn_decode_q4(*flat, seq_len=lens, q=q)
    for P, extra in ((16, 0), (64, 7), (512, 1)):
        mp = -(-L // P) + extra
        table = torch.randperm(B * mp, device=DEV)[:B * mp].reshape(B, mp).to(torch.int32)
        pool = _cache(B * mp, Hkv, P, d, k)
        sfa.sfa_kv_append_q4(kn, vn, torch.zeros(B, dtype=torch.int32, device=DEV), *pool, k=k, block_table=table)
        for _ in range(2):
            o2, lse2 = sfa.sfa_attn_decode_q4(*pool, block_table=table, seq_len=lens, q=q)
            assert torch.equal(o, o2) and torch.equal(lse, lse2)
        bad = table.clone()
        bad[2, 1:] = 1 << 29          # past the sequence's end: never read; clamped if it were
        o2, _ = sfa.sfa_attn_decode_q4(*pool, block_table=bad, seq_len=lens, q=q)
        assert torch.equal(o, o2)


def test_decode_q4_long_context():
    """Offsets past 32 bits in a long cache: one sequence of 2^21 keys and 12 KV heads of
    d = 256 (3.2 GB of values), the last keys against the oracle under a window."""
    L, Hkv, d, k = 1 << 21, 12, 256, 8
    cache = _cache(1, Hkv, L, d, k)
    for c in cache:
        c.zero_()
    T = 300
    kn = si.normal((1, Hkv, T, d), 9, "k", device=DEV)
    vn = si.normal((1, Hkv, T, d), 9, "v", device=DEV)
    lens = torch.tensor([L - T], dtype=torch.int32, device=DEV)
    sfa.sfa_kv_append_q4(kn, vn, lens, *cache, k=k)
    assert lens.tolist() == [L]
    q = si.normal((1, Hkv, d), 10, "q", device=DEV)
    qi, qv = sfa.sfa_topk_encode(q, k)
    o, lse = sfa.sfa_attn_decode_q4(*cache, q_idx=qi, q_val=qv, window=T)
    full, flse = sfa.sfa_attn_decode_q4(*cache, q=q)
    torch.cuda.synchronize()
    new = oracle.rows_q4(kn.cpu().numpy(), vn.cpu().numpy(), k)
    kv, vv = oracle.values_q4(*new[1:])
    O, E = oracle.attn_decode(qi.cpu().numpy(), qv.cpu().numpy(), new[0], kv, vv, d, 1 / math.sqrt(d))
    tol_o, tol_l = _bounds(qv.cpu().numpy(), kv, vv, 1 / math.sqrt(d), k, T)
    assert np.abs(np_f64(o) - O).max() <= tol_o * np.abs(vv).max()
    assert np.abs(np_f64(lse) - E).max() <= tol_l + 2.0 ** -20
    # the other L - T keys score 0 with value 0: the same numerator over l + (L - T)
    want = O * np.exp(E)[..., None] / (np.exp(E) + (L - T))[..., None]
    assert np.abs(np_f64(full) - want).max() <= 2 * tol_o * np.abs(vv).max()
    assert np.abs(np_f64(flse) - np.log(np.exp(E) + (L - T))).max() <= 1e-4


def test_q4_python_refusals():
    cache = _cache(2, 2, 64, 128, 16)
    q = torch.zeros((2, 4, 128), device=DEV)
    x = torch.zeros((2, 2, 3, 128), device=DEV)
    L = torch.zeros(2, dtype=torch.int32, device=DEV)
    slots = torch.zeros((2, 3), dtype=torch.int32, device=DEV)
    bad = list(cache)
    bad[4] = bad[4][..., :3].contiguous()
    for f in (lambda: sfa.sfa_attn_decode_q4(*bad, q=q), lambda: sfa.sfa_attn_decode_q4(*cache, q=q[:1]),
              lambda: sfa.sfa_attn_decode_q4(*cache, q=q, q_idx=q.int(), q_val=q),
              lambda: sfa.sfa_attn_decode_q4(*cache, q=q[..., :64].contiguous()),
              lambda: sfa.sfa_attn_decode_q4(*cache, q=q, seq_len=L[:1]),
              lambda: sfa.sfa_kv_append_q4(x, x, L, *cache, k=16, slots=slots),
              lambda: sfa.sfa_kv_append_q4(x, x, None, *cache, k=16, slots=slots[:1]),
              lambda: sfa.sfa_kv_append_q4(x, x, L, *cache, k=8),
              lambda: sfa.sfa_kv_append_q4(x, x[:1], L, *cache, k=16),
              lambda: sfa.sfa_kv_append_q4(x, x, L, *cache, k=16, v_out=x[:1].bfloat16())):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: sfa.sfa_kv_append_q4(x, x, L, *cache, k=16, v_out=x),
              lambda: sfa.sfa_kv_append_q4(x.half(), x, L, *cache, k=16),
              lambda: sfa.sfa_attn_decode_q4(cache[0].short(), *cache[1:], q=q)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(sfa.SfaError) as e:
        sfa.sfa_attn_decode_q4(*cache, q=q, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == sfa.SFA_ENOSPC
    with pytest.raises(sfa.SfaError) as e:
        sfa.sfa_attn_decode_q4(*cache, q=torch.zeros((2, 18, 128), device=DEV))
    assert e.value.status == sfa.SFA_ENOTSUP


@pytest.mark.parametrize("d,k", [(32, 8), (32, 32), (64, 16), (96, 24), (128, 16), (128, 128), (224, 40), (256, 256)])
def test_append_q4_of_ties(d, k):
    """Keys of one value, of zeros and of few values: the kept coordinates are
    sfa_topk_encode's, ties to the lower one."""
    g = torch.Generator().manual_seed(d + k)
    rows = torch.cat([torch.zeros(5, d), torch.full((5, d), -1.5), torch.randint(-2, 3, (60, d), generator=g).float()])
    n = rows.shape[0]
    kn = rows.to(DEV)[None, None].contiguous()
    cache = _cache(1, 1, n, d, k)
    sfa.sfa_kv_append_q4(kn, kn, torch.zeros(1, dtype=torch.int32, device=DEV), *cache, k=k)
    wi, _ = sfa.sfa_topk_encode(kn, k)
    assert torch.equal(cache[0].int(), wi.int())
