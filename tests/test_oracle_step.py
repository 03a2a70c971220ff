"""Pins of the oracle of the server's update (CPU): the 8-bit numbers are torch's e4m3 and e8m0, rounding at random is right in the
mean, the float64 step is torch's AdamW in float64, and the host side of the library: sizes, plans, refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import step as O


def test_codes_and_scales_are_torchs():
    code = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(code).view(torch.float8_e4m3fn).float().numpy()
    fine = (code & 127) != 127
    for s in (0, 1, 100, 127, 200, 246):
        got = O.decode(code, np.array([s], np.uint8))
        scale = torch.tensor([s], dtype=torch.uint8).view(torch.float8_e8m0fnu).double().item()
        assert scale == 2.0 ** (s - 127)
        assert np.array_equal(got[fine], (want.astype(np.float64) * scale).astype(np.float32)[fine])


@pytest.mark.parametrize("spread", [0.0, 3.0, 12.0])
def test_rounding_takes_one_of_the_two_neighbours_and_keeps_the_scale_small(spread):
    rng = np.random.default_rng(int(spread))
    x = (rng.standard_normal(256 * 64) * np.exp(rng.standard_normal(256 * 64) * spread)).astype(np.float32)
    x[:256] = 0.0
    x[256:300] = 0.0
    r = rng.integers(0, 65536, x.size)
    code, s = O.encode(x, r, False)
    val = O.decode(code, s).astype(np.float64)
    unit = np.repeat(2.0 ** (s.astype(np.float64) - 127), 256)
    y, v = np.abs(x.astype(np.float64)) / unit, np.abs(val) / unit
    assert y.max() <= 448 and (code & 127).max() <= 126
    # the top of every block is in the upper part of the range: half the scale would not hold it
    top = y.reshape(-1, 256).max(1)
    assert np.all((top >= 224) | (s == 0))
    below = O.E4M3[np.searchsorted(O.E4M3, y, side="right") - 1]
    above = O.E4M3[np.minimum(np.searchsorted(O.E4M3, y, side="left"), 126)]
    assert np.all((v == below) | (v == above))
    assert np.all((np.sign(val) == np.sign(x)) | (val == 0))
    exact = below == y
    assert np.array_equal(v[exact], y[exact])
    kept, _ = O.encode(np.abs(x), r, True)
    assert np.all((kept > 0) == (x != 0))


def test_rounding_is_right_in_the_mean():
    """65,536 roundings of one value with the 65,536 values of the random bits: the mean is the value, but for what 16 bits
    leave of the 20 that are cut off (half of 2^-16 of a step)."""
    rng = np.random.default_rng(3)
    x = np.zeros(256, np.float32)
    x[0] = 400.0
    x[1:] = np.exp(rng.uniform(np.log(2.0 ** -9), np.log(440.0), 255)).astype(np.float32)
    r = np.arange(65536)
    for i in range(1, 256, 5):
        lo = np.searchsorted(O.E4M3, float(x[i]), side="right") - 1
        gap = O.E4M3[lo + 1] - O.E4M3[lo]
        cut = math.floor((float(x[i]) - O.E4M3[lo]) / gap * 2 ** 20)
        ups = np.count_nonzero(cut + 16 * r + 8 >= 2 ** 20)
        # the rule above is what encode does ...
        for one in (0, 1000, 32768, 65535):
            code, s = O.encode(x, np.full(256, one), False)
            assert s[0] == 127 and code[i] == lo + (cut + 16 * one + 8 >= 2 ** 20)
        # ... and its mean is the value
        assert abs(O.E4M3[lo] + gap * ups / 65536 - float(x[i])) <= gap * 2.0 ** -17 * (1 + 1e-3) + gap * 2.0 ** -20


def test_random_bits_are_uniform_and_differ_with_seed_step_and_place():
    n = 1 << 18
    a = O.random16(0, n, 7, 1)
    assert np.array_equal(a[1000:2001], O.random16(1000, 1001, 7, 1))
    for other in (O.random16(0, n, 8, 1), O.random16(0, n, 7, 2), O.random16(0, n, 7 + (1 << 40), 1), np.roll(a, 1), np.roll(a, 2), np.roll(a, 256)):
        # correlation of independent uniform numbers: 0 with a deviation of n^-1/2; six of them
        c = np.corrcoef(a, other)[0, 1]
        assert abs(c) < 6 / math.sqrt(n)
    count = np.bincount(a >> 8, minlength=256)
    chi = np.sum((count - n / 256) ** 2 / (n / 256))
    assert abs(chi - 255) < 6 * math.sqrt(2 * 255)


def test_float64_step_is_torchs():
    rng = np.random.default_rng(5)
    p0 = rng.standard_normal(1000)
    p = torch.nn.Parameter(torch.from_numpy(p0.copy()))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    w, m, v = p0.copy(), np.zeros(1000), np.zeros(1000)
    for t in range(1, 6):
        g = rng.standard_normal(1000)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        m, v = 0.8 * m + 0.2 * g, 0.95 * v + 0.05 * g * g
        w, _, _ = O.weight64(w, m, v, t, 3e-3, 0.8, 0.95, 1e-6, 0.1)
        assert np.allclose(w, p.detach().numpy(), rtol=1e-13, atol=1e-13)


# ---- the library's host side ------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def B():
    from paper_2203_09044_amd import binding
    return binding


def rows(B, sizes, pbytes=4, gbytes=4, base=1 << 20, **kw):
    out, p, g = (B.StepTensor * len(sizes))(), base, base << 12
    for k, n in enumerate(sizes):
        out[k] = B.StepTensor(p, g, n, kw.get("lr_scale", 1.0), kw.get("weight_decay", 0.0))
        p += n * pbytes
        g += n * gbytes
    return out


SIZES = [1, 0, 255, 256, 257, 5000, 1024]


@pytest.mark.parametrize("bits,pt,gt", [(32, 0, 0), (32, 1, 0), (8, 0, 0), (8, 2, 1), (0, -1, 1)])
@pytest.mark.parametrize("sizes", [[1], [0, 0], SIZES, [5_000_001, 3, 4097]])
def test_plan_covers_every_element_once(B, bits, pt, gt, sizes):
    pb, gb = 4 if pt == 0 else 2, 4 if gt == 0 else 2
    t = rows(B, sizes, pb, gb)
    L = B.step_layout_of(t, pt, gt, bits)
    unit = 256 if bits == 8 else 1
    starts = np.concatenate([[0], np.cumsum([-(-n // unit) * unit for n in sizes])])
    assert L.elems == starts[-1] and L.blocks == (L.elems // 256 if bits == 8 else 0)
    assert L.chunk % 256 == 0 and L.partials >= 2
    plan = B.step_plan(t, L).numpy()
    assert plan.nbytes == L.plan_bytes
    assert L.plan_bytes == (40 * L.chunks or 16)
    entries = plan[:L.chunks * 40].view(np.dtype([("p", "<u8"), ("g", "<u8"), ("at", "<i8"), ("n", "<i4"), ("ls", "<f4"), ("wd", "<f4"), ("x", "<i4")]))
    k = 0
    for n, x, at in zip(sizes, t, starts):
        i = 0
        while i < n:                                # a piece ends at a multiple of its length, or with its tensor
            e = entries[k]
            assert e["g"] == x.grad + i * gb and e["at"] == at + i and e["n"] == min(L.chunk - (at + i) % L.chunk, n - i)
            assert e["p"] == (x.param + i * pb if bits else 0)
            i += int(e["n"])
            k += 1
    assert k == len(entries)


def test_layout_refusals(B):
    ok = rows(B, SIZES)
    for bad in ((3, 0, 32), (0, 3, 32), (-1, 0, 32), (0, 0, 16), (0, 0, 0), (0, -1, 32)):
        with pytest.raises(B.Co3Error):
            B.step_layout_of(ok, *bad)
    for field, value in (("n", -1), ("n", (1 << 33) + 1), ("lr_scale", -1.0), ("lr_scale", math.nan), ("weight_decay", math.inf),
                         ("param", 0), ("grad", 0), ("param", 4098), ("grad", 4098)):
        t = rows(B, SIZES)
        setattr(t[3], field, value)
        with pytest.raises(B.Co3Error):
            B.step_layout_of(t, 0, 0, 32)
    t = rows(B, [0, 5])
    t[0].param = t[0].grad = 0                     # a tensor of no elements has no address
    B.step_layout_of(t, 0, 0, 8)
    with pytest.raises(B.Co3Error):                 # together too long
        B.step_layout_of(rows(B, [1 << 32, 1 << 32, 1], 2, 2), 1, 1, 32)
    assert B._lib.co3_step_layout_of(None, 1, 0, 0, 32, C.byref(B.StepLayout())) == B.EINVAL
    assert B._lib.co3_step_layout_of(ok, 0, 0, 0, 32, C.byref(B.StepLayout())) == B.EINVAL


def test_plan_refusals(B):
    t = rows(B, SIZES)
    L = B.step_layout_of(t, 0, 0, 32)
    for field in ("elems", "chunks", "chunk", "partials", "plan_bytes"):
        W = B.StepLayout.from_buffer_copy(L)
        setattr(W, field, getattr(W, field) + 8)
        with pytest.raises(B.Co3Error):
            B.step_plan(t, W)
    buf = np.zeros(L.plan_bytes // 8, np.int64)
    assert B._lib.co3_step_plan(t, len(t), C.byref(L), C.c_void_p(buf.ctypes.data), L.plan_bytes - 1) == B.EINVAL
    assert B._lib.co3_step_plan(t, len(t), C.byref(L), None, L.plan_bytes) == B.EINVAL
    # the same parameter twice, one inside another, a parameter on a gradient; the same gradient twice is fine
    for change in ({"param": t[5].param}, {"param": t[5].param + 4}, {"param": t[4].grad}, {"grad": t[5].param + 400}):
        w = rows(B, SIZES)
        setattr(w[3], *list(change.items())[0])
        with pytest.raises(B.Co3Error):
            B.step_plan(w, L)
    w = rows(B, SIZES)
    w[3].grad = w[5].grad
    B.step_plan(w, L)


def test_device_calls_refuse_bad_arguments_on_the_host(B):
    """Checked before anything is launched (safe without a GPU): the addresses are never touched."""
    t = rows(B, SIZES)
    L32, L8, L0 = B.step_layout_of(t, 0, 0, 32), B.step_layout_of(t, 0, 0, 8), B.step_layout_of(t, -1, 0, 0)
    p, lib = C.c_void_p(1 << 20), B._lib
    odd = C.c_void_p((1 << 20) + 2)
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, max_norm=1.0, t=1, seed=0)
    args = lambda **kw: C.byref(B.AdamwArgs(**{**good, **kw}))  # noqa: E731
    bad = [dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan),
           dict(eps=0.0), dict(eps=1e-60), dict(eps=1e-39), dict(eps=math.nan), dict(grad_scale=0.0), dict(grad_scale=math.inf), dict(grad_scale=1e-39), dict(grad_scale=1e39), dict(grad_scale=-1.0),
           dict(max_norm=0.0), dict(max_norm=math.nan), dict(t=0)]
    for kw in bad:
        assert lib.co3_adamw(C.byref(L32), p, None, p, p, args(**kw), None, None) == B.EINVAL, kw
        assert lib.co3_adamw8(C.byref(L8), p, None, p, p, p, p, args(**kw), None, None) == B.EINVAL, kw
        if "t" not in kw:
            assert lib.co3_step_begin(args(**kw), None, 0, None, p, None) == B.EINVAL, kw
            assert lib.co3_adamw_clipped(C.byref(L32), p, None, p, p, args(**kw), None, p, p, None) == B.EINVAL, kw
            assert lib.co3_adamw8_clipped(C.byref(L8), p, None, p, p, p, p, args(**kw), None, p, p, None) == B.EINVAL, kw
    for a in ((None, p, None, p, p), (C.byref(L32), None, None, p, p), (C.byref(L8), p, None, p, p), (C.byref(L0), p, None, p, p),
              (C.byref(L32), p, p, p, p), (C.byref(L32), p, None, None, p), (C.byref(L32), p, None, p, None),
              (C.byref(L32), p, None, odd, p), (C.byref(L32), odd, None, p, p)):
        assert lib.co3_adamw(*a, args(), None, None) == B.EINVAL
    assert lib.co3_adamw(C.byref(L32), p, None, p, p, None, None, None) == B.EINVAL
    assert lib.co3_adamw(C.byref(L32), p, None, p, p, args(), odd, None) == B.EINVAL
    for a in ((p, None, p, p), (p, p, None, p), (p, p, p, None), (None, p, p, p), (odd, p, p, p)):
        assert lib.co3_adamw8(C.byref(L8), p, None, *a, args(), None, None) == B.EINVAL
    assert lib.co3_adamw8(C.byref(L32), p, None, p, p, p, p, args(), None, None) == B.EINVAL
    for a in ((C.byref(L0), p, 1.0, 1.0, None, p), (C.byref(L0), p, 1.0, 1.0, p, None), (C.byref(L0), p, 0.0, 1.0, p, p),
              (C.byref(L0), p, 1.0, 0.0, p, p), (C.byref(L0), p, math.nan, 1.0, p, p), (C.byref(L0), p, 1.0, math.nan, p, p),
              (None, p, 1.0, 1.0, p, p), (C.byref(L0), None, 1.0, 1.0, p, p), (C.byref(L0), p, 1.0, 1.0, p, odd)):
        assert lib.co3_grad_norm(*a, None) == B.EINVAL
    for a in ((None, p, p), (odd, p, p), (p, None, p), (p, odd, p)):          # partials, state, moments
        assert lib.co3_adamw_clipped(C.byref(L32), p, None, a[2], a[2], args(), None, a[0], a[1], None) == B.EINVAL
        assert lib.co3_adamw8_clipped(C.byref(L8), p, None, p, p, p, p, args(), None, a[0], a[1], None) == B.EINVAL
    assert lib.co3_adamw_clipped(C.byref(L32), p, None, p, p, args(), odd, p, p, None) == B.EINVAL
    assert lib.co3_adamw_clipped(C.byref(L8), p, None, p, p, args(), None, p, p, None) == B.EINVAL
    assert lib.co3_adamw_clipped(C.byref(L32), p, p, p, p, args(), None, p, p, None) == B.EINVAL
    assert lib.co3_adamw_clipped(None, p, None, p, p, args(), None, p, p, None) == B.EINVAL
    assert lib.co3_adamw8_clipped(C.byref(L8), p, None, p, None, p, p, args(), None, p, p, None) == B.EINVAL
    assert lib.co3_grad_sumsq(C.byref(L0), p, None, None) == B.EINVAL
    for a in ((args(), None, 0, None, None), (args(), None, -1, None, p), (args(), odd, 1, None, p), (args(), None, 0, odd, p),
              (args(), None, 0, None, odd), (None, None, 0, None, p)):
        assert lib.co3_step_begin(*a, None) == B.EINVAL


def test_handles_refuse_what_they_cannot_serve():
    from paper_2203_09044_amd import AdamW, GradNorm
    x = torch.zeros(8)
    with pytest.raises(ValueError):
        AdamW([x], [x.clone()])                      # not on a GPU
    with pytest.raises(ValueError):
        GradNorm([])
    for kw in (dict(state_bits=16), dict(betas=(1.0, 0.9)), dict(eps=0.0), dict(max_norm=0.0), dict(grad_scale=0.0)):
        with pytest.raises(ValueError):
            AdamW([x], [x.clone()], **kw)
    with pytest.raises(ValueError):
        GradNorm([x], max_norm=-1.0)
