"""GPU parity of the rotary positions: sfa_rope, sfa_rope_encode and its
straight-through backward against the float64 oracle.

Tolerance (derived): cosine and sine are float32 roundings of exact values, off by
2^-25 each, so a rotated value is off by 2^-25 (|x1| + |x2|) before its own rounding of
2^-24 |y|; a bf16 result adds half a step, 2^-8 |y|.  2^-40 of both terms stands for
the float64 arithmetic before."""
import numpy as np
import pytest
import torch

import oracle
import paper_2603_22300_amd as sfa
import sfa_inputs as si

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _bound(x, y, rot, pairing, bf16, f32=False):
    u, v = oracle.rope_pairs(rot, pairing)
    mag = np.zeros_like(y)
    m = np.abs(x[..., u]) + np.abs(x[..., v])
    mag[..., u], mag[..., v] = m, m
    # f32: one of the two products is itself rounded to float32 (half a step, 2^-24 of at
    # most |x1| or |x2|, as |sin| and |cos| are at most 1), the other enters an fma exactly
    w = 2.0 ** -25 + f32 * 2.0 ** -24
    return ((w * mag + 2.0 ** -24 * np.abs(y)) * (1 + 2.0 ** -15) + 2.0 ** -8 * np.abs(y) * bf16 + 1e-45)


def _positions(A, B, n, seed, far):
    rng = np.random.default_rng(seed)
    pos = rng.integers(-far if far > 1000 else 0, far + 1, (A, B, n)).astype(np.int32)
    if far > 2 ** 30:
        pos[0, 0, 0], pos[-1, -1, -1] = 2 ** 31 - 1, -2 ** 31
    return pos


CASES = [  # B, H, n, d, sections, pairing, order, far
    (2, 3, 37, 128, (16, 24, 24), "halves", "sections", 4000),
    (1, 1, 1, 128, (64,), "halves", "sections", 2 ** 31 - 1),
    (3, 5, 66, 64, (8, 12, 12), "halves", "interleaved", 100000),
    (1, 2, 130, 256, (64, 64), "neighbours", "own", 512),
    (2, 4, 19, 96, (12, 12), "neighbours", "own", 300),      # half of each head turns
    (1, 3, 33, 80, (20, 8), "halves", "interleaved", 2 ** 20),
    (2, 2, 9, 7, (1, 2), "neighbours", "sections", 50),       # odd d: single elements
    (1, 2, 5, 2, (1,), "halves", "sections", 9),
    (1, 2, 70, 250, (100, 20, 3, 2), "halves", "sections", 70000),
    (1, 2, 3, 255, (127,), "neighbours", "sections", 70000),
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_rope(case, xt, yt):
    B, H, n, d, sections, pairing, order, far = case
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = si.normal((B, H, n, d), d + n, "x", device=DEV).to(types[xt])
    pos = _positions(len(sections), B, n, n, far)
    plan = sfa.sfa_rope_plan(d, sections, theta=1e4, pairing=pairing, order=order)
    axis, freq = oracle.rope_ladder(sections, 1e4, order)
    for inverse in (False, True):
        y = sfa.sfa_rope(x, torch.from_numpy(pos).to(DEV), plan, inverse=inverse, y_dtype=types[yt])
        torch.cuda.synchronize()
        x64 = x.double().cpu().numpy()
        want = oracle.rope(x64, pos, axis, np.array(plan.freq), pairing, inverse)
        err = np.abs(y.double().cpu().numpy() - want)
        bound = _bound(x64, want, plan.rot, pairing, yt == "bf16")
        assert (err <= bound).all(), (err / bound).max()
        assert np.array_equal(y[..., plan.rot:].float().cpu().numpy(),
                              x[..., plan.rot:].to(types[yt]).float().cpu().numpy())  # copied


def test_rope_views_shared_positions_and_in_place():
    """A view of a packed projection in and out, positions shared by the axes and by the
    sequences, unaligned views, and y = x."""
    B, H, n, d = 2, 3, 21, 64
    plan = sfa.sfa_rope_plan(d, (16, 16))
    packed = si.normal((B, n, H + 2, d), 5, "x", device=DEV).to(torch.bfloat16)
    x = packed[:, :, 1:H + 1].transpose(1, 2)
    at = torch.arange(n, dtype=torch.int32, device=DEV)
    full = at.expand(2, B, n).contiguous()
    want = sfa.sfa_rope(x.contiguous(), full, plan)
    for pos in (at, at.expand(B, n), full, at.reshape(1, 1, n)):
        assert torch.equal(sfa.sfa_rope(x, pos, plan), want)
    out = torch.full((B, n, H + 1, d), 7.0, dtype=torch.bfloat16, device=DEV)
    sfa.sfa_rope(x, at, plan, y=out[:, :, :H].transpose(1, 2))
    assert torch.equal(out[:, :, :H].transpose(1, 2), want) and bool((out[:, :, H] == 7).all())
    store = torch.empty(B * H * n * d + 1, dtype=torch.bfloat16, device=DEV)
    odd = store[1:].view(B, H, n, d)
    odd.copy_(x)
    assert torch.equal(sfa.sfa_rope(odd, at, plan), want)
    sfa.sfa_rope(odd, at, plan, y=odd)
    assert torch.equal(odd, want)
    keep = packed[:, :, 0].clone(), packed[:, :, H + 1].clone()
    sfa.sfa_rope(x, at, plan, y=x)
    assert torch.equal(x, want) and torch.equal(packed[:, :, 0], keep[0]) and torch.equal(packed[:, :, H + 1], keep[1])
    empty = torch.empty((B, H, 0, d), device=DEV)
    assert sfa.sfa_rope(empty, at[:0], plan).shape == (B, H, 0, d)


FORMATS = [(torch.int32, torch.float32), (torch.int16, torch.bfloat16), (torch.uint8, torch.float16),
           (torch.int16, torch.float32)]


@pytest.mark.parametrize("case,k", [(c, k) for c in CASES for k in sorted({1, min(16, c[3]), c[3]})])
@pytest.mark.parametrize("bf16", [False, True])
def test_rope_encode_is_the_code_of_the_rotated_row(case, k, bf16):
    """Bit for bit the coding kernel's code of sfa_rope's float32 rows (which test_rope
    bounds), whose selection the oracle confirms; every format pair in turn."""
    B, H, n, d, sections, pairing, order, far = case
    x = si.normal((B, H, n, d), d + k, "x", device=DEV)
    if bf16:
        x = x.to(torch.bfloat16)
    strided = torch.zeros((B, n, H + 1, d), dtype=x.dtype, device=DEV)
    view = strided[:, :, :H].transpose(1, 2)
    view.copy_(x)
    pos = torch.from_numpy(_positions(len(sections), B, n, k, far)).to(DEV)
    plan = sfa.sfa_rope_plan(d, sections, theta=1e6, pairing=pairing, order=order)
    y = sfa.sfa_rope(x, pos, plan, y_dtype=torch.float32)
    it, vt = FORMATS[(d + k + n) % 4]
    want = sfa.sfa_topk_encode(y, k, idx_dtype=it, val_dtype=vt)
    for src in (x, view):
        got = sfa.sfa_rope_encode(src, pos, plan, k, idx_dtype=it, val_dtype=vt)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    oi, _ = oracle.topk_encode(y.cpu().numpy(), k)
    assert np.array_equal(got[0].cpu().numpy().astype(np.int64), oi)


def test_rope_encode_many_tokens_and_heads():
    """Past the persistent grid: several tokens a wavefront, and slices of heads."""
    plan = sfa.sfa_rope_plan(64, (32,))
    for B, H, n in ((1, 2, 20000), (2, 31, 700), (4000, 33, 1)):
        x = si.normal((B, H, n, 64), n, "x", device=DEV).to(torch.bfloat16)
        pos = torch.randint(0, 1 << 20, (B, n), dtype=torch.int32, device=DEV)
        y = sfa.sfa_rope(x, pos, plan, y_dtype=torch.float32)
        want = sfa.sfa_topk_encode(y, 8)
        got = sfa.sfa_rope_encode(x, pos, plan, 8)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("case,k", [(c, k) for c in CASES for k in sorted({1, min(16, c[3]), c[3]})])
@pytest.mark.parametrize("bf16", [False, True])
def test_rope_encode_bwd(case, k, bf16):
    """Against the formula, and against differences of the loss sum(g * val): the code
    values are linear in x on a fixed support, so the central difference in float64
    along any direction is <dx, direction>."""
    B, H, n, d, sections, pairing, order, far = case
    x = si.normal((B, H, n, d), d + k, "x", device=DEV)
    pos = _positions(len(sections), B, n, k, far)
    plan = sfa.sfa_rope_plan(d, sections, theta=1e4, pairing=pairing, order=order)
    freq, axis = np.array(plan.freq), np.array(plan.axis)
    pt = torch.from_numpy(pos).to(DEV)
    idx, _ = sfa.sfa_rope_encode(x, pt, plan, k, idx_dtype=[torch.int32, torch.int16, torch.uint8][k % 3])
    g = si.normal((B, H, n, k), d, "g", device=DEV)
    packed = torch.full((B, n, H + 1, d), 3.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
    dx = packed[:, :, 1:].transpose(1, 2)
    sfa.sfa_rope_encode_bwd(idx, g, pt, plan, dx=dx)
    torch.cuda.synchronize()
    assert bool((packed[:, :, 0] == 3).all())
    dense = np.zeros((B, H, n, d))
    np.put_along_axis(dense, idx.long().cpu().numpy(), g.double().cpu().numpy(), -1)
    want = oracle.rope(dense, pos, axis, freq, pairing, inverse=True)
    got = dx.double().cpu().numpy()
    bound = _bound(dense, want, plan.rot, pairing, bf16, f32=True)
    assert (np.abs(got - want) <= bound).all()
    assert torch.equal(sfa.sfa_rope_encode_bwd(idx, g, pt, plan, dx_dtype=packed.dtype), dx)
    rng = np.random.default_rng(k)
    v, x64 = rng.standard_normal(x.shape), x.double().cpu().numpy()
    loss = lambda z: float((g.double().cpu().numpy() * np.take_along_axis(  # noqa: E731
        oracle.rope(z, pos, axis, freq, pairing), idx.long().cpu().numpy(), -1)).sum())
    diff = (loss(x64 + 0.5 * v) - loss(x64 - 0.5 * v))
    slack = float((bound * np.abs(v)).sum()) + 1e-9 * float(np.abs(got * v).sum())
    assert abs(diff - float((got * v).sum())) <= slack


def test_rope_python_refusals():
    plan = sfa.sfa_rope_plan(64, (8, 8))
    x = torch.zeros((2, 3, 4, 64), device=DEV)
    pos = torch.zeros((2, 2, 4), dtype=torch.int32, device=DEV)
    for a in ((x[..., ::2], pos), (x[0], pos), (x[..., :32], pos), (x, pos[:, :, :3]), (x, pos[:, :, ::2]),
              (x, pos.expand(2, 2, 4).repeat(1, 2, 1)), (x, torch.zeros((3, 2, 4), dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            sfa.sfa_rope(a[0], a[1], plan)
    for bad in ((x.half(), pos), (x, pos.long())):
        with pytest.raises(TypeError):
            sfa.sfa_rope(*bad, plan)
    with pytest.raises(sfa.SfaError):
        sfa.sfa_rope(x, pos, plan, y=torch.zeros((1, 1, 1, 64), device=DEV).expand(2, 3, 4, 64))
    with pytest.raises(ValueError):
        sfa.sfa_rope(x, pos, plan, y=x[:1])
    with pytest.raises(sfa.SfaError):
        sfa.sfa_rope_encode(x, pos, plan, 65)


def test_rope_of_more_blocks_than_one_grid_dimension():
    """Millions of tokens one element at a time (rows that start off any boundary of four):
    the first, middle and last tokens are those of a call on them alone."""
    d, n, k = 256, (1 << 22) + 5, 8
    plan = sfa.sfa_rope_plan(d, theta=1e4)
    x = torch.zeros((1, 1, n, d + 1), dtype=torch.bfloat16, device=DEV)[..., :d]
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    idx = torch.zeros((1, 1, n, k), dtype=torch.uint8, device=DEV)
    g = torch.zeros((1, 1, n, k), device=DEV)
    spans = [slice(0, 7), slice(1 << 21, (1 << 21) + 9), slice(n - 6, n)]
    for i, s in enumerate(spans):
        x[:, :, s] = torch.randn(x[:, :, s].shape, generator=torch.Generator().manual_seed(i)).to(DEV, torch.bfloat16)
        g[:, :, s] = torch.randn(g[:, :, s].shape, generator=torch.Generator().manual_seed(9 + i)).to(DEV)
        idx[:, :, s] = torch.arange(k, dtype=torch.uint8, device=DEV) * 31
    y = sfa.sfa_rope(x, pos, plan)
    ci, cv = sfa.sfa_rope_encode(x, pos, plan, k, idx_dtype=torch.uint8, val_dtype=torch.float16)
    dx = torch.empty((1, 1, n, d + 1), dtype=torch.bfloat16, device=DEV)[..., :d]
    sfa.sfa_rope_encode_bwd(idx, g, pos, plan, dx=dx)
    for s in spans:
        part = x[:, :, s].contiguous()
        assert torch.equal(y[:, :, s], sfa.sfa_rope(part, pos[s], plan))
        pi, pv = sfa.sfa_rope_encode(part, pos[s], plan, k, idx_dtype=torch.uint8, val_dtype=torch.float16)
        assert torch.equal(ci[:, :, s], pi) and torch.equal(cv[:, :, s], pv)
        pd = sfa.sfa_rope_encode_bwd(idx[:, :, s].contiguous(), g[:, :, s].contiguous(), pos[s].contiguous(), plan,
                                     dx_dtype=torch.bfloat16)
        assert torch.equal(dx[:, :, s], pd)


@pytest.mark.parametrize("d", [2, 48, 64, 96, 128, 200, 256])
def test_rope_encode_of_ties(d):
    """Rows of one value, of zeros, of few values, with infinities and NaN, at k from 1 to d:
    the code is sfa_topk_encode's of the rotated rows, ties to the lower coordinate."""
    g = torch.Generator().manual_seed(d)
    rows = [torch.zeros(9, d), torch.full((9, d), -1.5), torch.randint(-2, 3, (40, d), generator=g).float(),
            torch.randint(0, 2, (20, d), generator=g).float() * 2.0 ** -140, torch.randn(30, d, generator=g)]
    odd = torch.randn(20, d, generator=g)
    odd[:, 0] = float("inf")
    odd[::3, d // 2] = float("nan")
    x = torch.cat(rows + [odd]).to(DEV)[None, None].repeat(1, 3, 1, 1).contiguous()
    pos = torch.zeros(x.shape[2], dtype=torch.int32, device=DEV)
    pos[::2] = 77
    for pairing in ("halves", "neighbours"):
        plan = sfa.sfa_rope_plan(d, theta=1e4, pairing=pairing)
        y = sfa.sfa_rope(x, pos, plan)
        for k in sorted({1, 2, min(d, 16), d // 2, d - 1, d}):
            i, v = sfa.sfa_rope_encode(x, pos, plan, k)
            wi, wv = sfa.sfa_topk_encode(y, k)
            assert torch.equal(i, wi) and torch.equal(v.view(torch.int32), wv.view(torch.int32)), (pairing, k)
