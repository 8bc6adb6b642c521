"""Oracle of the rotary positions, the page tables and the 4-bit cache (numpy,
float64; plain loops where the definition is sequential)."""
from __future__ import annotations

import numpy as np

from .sfa_oracle import bf16_rne, topk_encode, widen


def rope_pairs(rot: int, pairing: str):
    """The two coordinates of each pair."""
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if pairing == "halves" else (2 * i, 2 * i + 1)


def rope_ladder(sections, theta: float, order: str):
    """(axis, frequency) of each pair."""
    axis, freq = [], []
    if order == "interleaved":
        left, a = list(sections), 0
        while sum(left):
            if left[a]:
                axis.append(a)
                left[a] -= 1
            a = (a + 1) % len(left)
    else:
        for a, m in enumerate(sections):
            axis += [a] * m
    half = sum(sections)
    for i, a in enumerate(axis):
        if order == "own":
            freq.append(float(theta) ** (-(i - sum(sections[:a])) / sections[a]))
        else:
            freq.append(float(theta) ** (-2.0 * i / (2 * half)))
    return np.array(axis), np.array(freq)


def rope(x, pos, axis, freq, pairing: str, inverse: bool = False) -> np.ndarray:
    """x [B, H, n, d] (any real) turned by pos [naxes, B, n]; float64 throughout, no
    rounding of the cosines."""
    y = np.array(x, dtype=np.float64)
    u, v = rope_pairs(2 * len(axis), pairing)
    ang = np.stack([np.asarray(pos, np.float64)[a] * f for a, f in zip(axis, freq)], -1)[:, None]
    c, s = np.cos(ang), np.sin(ang) * (-1.0 if inverse else 1.0)
    a, b = y[..., u].copy(), y[..., v].copy()
    y[..., u], y[..., v] = a * c - b * s, b * c + a * s
    return y


def page_tables(old, new, table, free, free_in: int, P: int, num_pages: int, n_rows: int):
    """sfa_page_tables as a list of steps: every sequence gives back, then every
    sequence takes.  table and free are changed in place; returns (got, free_out,
    starts, slots, pos)."""
    B, mp = table.shape
    cap = mp * P
    clamp = lambda v: max(0, min(int(v), cap))  # noqa: E731
    old, new = [clamp(v) for v in old], [clamp(v) for v in new]
    pages = lambda n: -(-n // P)  # noqa: E731
    stack = [int(v) for v in free[:max(0, min(int(free_in), num_pages))]]
    given = len(stack)
    for b in range(B):
        for j in range(pages(new[b]), pages(old[b])):
            if len(stack) < num_pages:
                stack.append(int(table[b, j]))
    got, starts, slots, pos = [], [0], np.full(n_rows, -1), np.full(n_rows, -1)
    for b in range(B):
        have = pages(old[b])
        while have < pages(new[b]) and stack:
            table[b, have] = stack.pop()
            have += 1
        reach = new[b] if new[b] <= old[b] else min(new[b], have * P)
        got.append(reach)
        for t in range(max(0, new[b] - old[b])):
            r, p = starts[-1] + t, old[b] + t
            if r < n_rows:
                pos[r] = p
                if p < reach and 0 <= table[b, p // P] < num_pages:
                    slots[r] = table[b, p // P] * P + p % P
        starts.append(starts[-1] + max(0, new[b] - old[b]))
    for i in range(given, len(stack)):
        free[i] = stack[i]
    return np.array(got), len(stack), np.array(starts), slots, pos


def quant_q4(x: np.ndarray, bf16_scale: bool = False):
    """Signed 4-bit rows of x [..., m] (float32): s = max|x| / 7 (a float32 division;
    bf16_scale: rounded to nearest-even bfloat16), q = x / s (a float32 division)
    rounded half to even, within [-7, 7]; s = 0: q = 0.  Returns (q int8, s float32)."""
    x = np.asarray(x, dtype=np.float32)
    s = (np.abs(x).max(axis=-1) / np.float32(7)).astype(np.float32)
    if bf16_scale:
        s = widen(bf16_rne(s)).astype(np.float32)
    safe = np.where(s > 0, s, np.float32(1)).astype(np.float32)
    q = np.clip(np.rint((x / safe[..., None]).astype(np.float32)), -7, 7)
    return np.where(s[..., None] > 0, q, 0).astype(np.int8), s


def pack_q4(q: np.ndarray) -> np.ndarray:
    """Two numbers to a byte in two's complement, the first in the low half."""
    u = np.asarray(q, dtype=np.int64) % 16
    return (u[..., 0::2] + 16 * u[..., 1::2]).astype(np.uint8)


def unpack_q4(b: np.ndarray) -> np.ndarray:
    b = np.asarray(b, dtype=np.int64)
    u = np.stack((b % 16, b // 16), -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))
    return np.where(u >= 8, u - 16, u).astype(np.int8)


def rows_q4(k_new: np.ndarray, v_new: np.ndarray, k: int):
    """The 4-bit cache's five fields of key and value rows [..., d] (float32): (idx,
    packed code values, their scale, packed values, their scales as float32)."""
    ci, cv = topk_encode(k_new, k)
    kq, ks = quant_q4(cv)
    vq, vs = quant_q4(v_new.reshape(v_new.shape[:-1] + (-1, 32)), bf16_scale=True)
    return ci, pack_q4(kq), ks, pack_q4(vq.reshape(v_new.shape)), vs


def values_q4(kc_val, kc_scale, v_cache, v_scale):
    """What a 4-bit cache stands for: code values [..., k] and value rows [..., d], float64."""
    kv = unpack_q4(kc_val).astype(np.float64) * np.asarray(kc_scale, np.float64)[..., None]
    v = unpack_q4(v_cache).astype(np.float64)
    return kv, v * np.repeat(np.asarray(v_scale, np.float64), 32, axis=-1)
