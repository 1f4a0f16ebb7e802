"""Rotary positions against the 64-bit oracle.

The bound of an element r of a pair (p, q), amplitude a: sine and cosine are off by 2^-23 (angle, polynomial and its steps), their
product with the amplitude, the second product and the fused sum by 2^-24 each: 3 * 2^-23 a (|p| + |q|); the 64-bit angle by 4 * 2^-53 of
itself; then the output's own rounding.
"""
import math

import numpy as np
import pytest

from gpu_util import say, torch_cuda
from test_gpu_kv import DT, U_OUT

pytestmark = pytest.mark.gpu


def _km():
    import paper_2608_14648_amd as km
    return km


def _bound(x, want, pos, freq, dims, layout, type_, amp=1.0):
    i = np.arange(dims // 2)
    a, b = (i, i + dims // 2) if layout == "halves" else (2 * i, 2 * i + 1)
    size = np.zeros_like(x)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    ang = np.zeros(x.shape[2])
    ang[a] = ang[b] = np.abs(freq)
    far = np.abs(np.asarray(pos, np.float64))[:, None, None] * ang
    step = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}[type_]  # below the least normal number
    return amp * size * (3 * 2.0 ** -23 + 4 * 2.0 ** -53 * far) + U_OUT[type_] * np.abs(want) * (1 + 2.0 ** -20) + step


def _check(got, x, pos, freq, dims, layout, type_, inverse=False, amp=1.0, label=""):
    import oracle.kv_ops as ops
    x, got = (t.float().cpu().numpy().astype(np.float64) for t in (x, got))
    want = ops.rotate(x, pos, freq, dims, layout, inverse, amp)
    bad = np.abs(got - want) - _bound(x, want, pos, freq, dims, layout, type_, amp)
    assert bad.max() <= 0, f"{label}: {np.abs(got - want).flat[bad.argmax()]:.3e} at {np.unravel_index(bad.argmax(), bad.shape)}"
    if dims < x.shape[2]:
        np.testing.assert_array_equal(got[..., dims:], x[..., dims:], err_msg=label)


def _rows(torch, rng, shape, type_):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(getattr(torch, DT[type_])).cuda()


CASES = [
    # d, dims, q_heads, k_heads, lens, rows
    (128, 128, 8, 2, [1], [1]),
    (128, 64, 5, 1, [700, 3, 0, 90], [1, 3, 0, 17]),
    (64, 64, 2, 2, [9000, 50], [600, 50]),
    (80, 20, 3, 1, [40, 7], [9, 7]),
    (96, 24, 1, 3, [131072, 2 ** 30], [2, 1]),
    (16, 2, 1, 1, [5], [5]),
    (256, 256, 2, 1, [33], [30]),
    (48, 44, 2, 1, [33, 12], [30, 1]),
    (128, 6, 4, 0, [1200], [1100]),
]


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rotate(case, layout, type_):
    torch, km = torch_cuda(), _km()
    d, dims, hq, hk, lens, rows = CASES[case]
    say(f"kv_rotate {type_} {layout} d={d} dims={dims} heads={hq}+{hk} lens={lens} rows={rows}")
    rng = np.random.default_rng(300 + case)
    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    total = int(starts[-1])
    pos = np.concatenate([np.arange(l - r, l) for l, r in zip(lens, rows)])
    q = _rows(torch, rng, (total, hq, d), type_)
    k = _rows(torch, rng, (total, hk, d), type_) if hk else None
    amp = 1.0 if case % 2 else 1.25
    rot = km.kv_rotary(dims, 10000.0, layout, amplitude=amp)
    freq = 10000.0 ** (-2.0 * np.arange(dims // 2) / dims)
    np.testing.assert_allclose(rot.freq.cpu().numpy(), freq, rtol=1e-14)
    seqs = km.KvSeqs(torch.zeros((len(lens), 1), dtype=torch.int32, device="cuda"),
                     torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.from_numpy(starts).cuda(), rows=total,
                     max_rows=max(rows))
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    for inverse in (False, True):
        a, b = km.kv_rotate(rot, seqs, q, k, inverse=inverse)
        _check(a, q, pos, freq, dims, layout, type_, inverse, amp, "queries")
        if hk:
            _check(b, k, pos, freq, dims, layout, type_, inverse, amp, "keys")
        # the same by positions, and in place
        c, e = km.kv_rotate(rot, at, q, k, inverse=inverse)
        assert torch.equal(a, c) and (k is None or torch.equal(b, e))
        q2, k2 = q.clone(), None if k is None else k.clone()
        r, s = km.kv_rotate(rot, seqs, q2, k2, inverse=inverse, q_out=q2, k_out=k2)
        assert r is q2 and s is k2 and torch.equal(a, q2) and (k is None or torch.equal(b, k2))


def test_any_position():
    """Positions of either sign up to the ends of 32 bits, in any order."""
    torch, km = torch_cuda(), _km()
    pos = np.array([0, -1, 1, 2 ** 31 - 1, -2 ** 31, 12345678, 7, 7, -5, 1 << 20], np.int64)
    rng = np.random.default_rng(5)
    x = _rows(torch, rng, (len(pos), 3, 64), "f32")
    rot = km.kv_rotary(64)
    got, none = km.kv_rotate(rot, torch.from_numpy(pos.astype(np.int32)).cuda(), x)
    assert none is None
    _check(got, x, pos, 10000.0 ** (-np.arange(32) / 32.0), 64, "halves", "f32")


@pytest.mark.parametrize("scaling", ["linear", "base", "parts"])
def test_scaled_frequencies(scaling):
    torch, km = torch_cuda(), _km()
    dims, factor, original = 64, 8.0, 4096
    f = 10000.0 ** (-2.0 * np.arange(dims // 2) / dims)
    got = km.kv_rotary(dims, scaling=scaling, factor=factor, original=original).freq.cpu().numpy()
    if scaling == "linear":
        want = f / factor
    elif scaling == "base":
        want = (10000.0 * factor ** (dims / (dims - 2))) ** (-2.0 * np.arange(dims // 2) / dims)
        assert got[0] == 1.0 and abs(got[-1] / f[-1] - 1 / factor) < 1e-12
    else:
        keep = np.clip((original * f / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        want = f * keep + f / factor * (1 - keep)
        assert got[0] == f[0] and got[-1] == f[-1] / factor
    np.testing.assert_allclose(got, want, rtol=1e-13)


def test_rows_inside_a_projection_turned_in_place():
    """Queries and keys side by side in one buffer, turned where they lie; the values between them stay."""
    torch, km = torch_cuda(), _km()
    rng = np.random.default_rng(6)
    for type_ in ("bf16", "f32"):
        fused = _rows(torch, rng, (70, 8 + 2 + 2, 128), type_)
        was = fused.clone()
        seqs = km.KvSeqs(torch.zeros((2, 1), dtype=torch.int32, device="cuda"),
                         torch.tensor([60, 1000], dtype=torch.int32, device="cuda"),
                         torch.tensor([0, 60, 70], dtype=torch.int32, device="cuda"), rows=70, max_rows=60)
        q, k = fused[:, :8], fused[:, 10:]
        want = km.kv_rotate(km.kv_rotary(128), seqs, was[:, :8], was[:, 10:])
        km.kv_rotate(km.kv_rotary(128), seqs, q, k, q_out=q, k_out=k)
        assert torch.equal(fused[:, :8], want[0]) and torch.equal(fused[:, 10:], want[1])
        assert torch.equal(fused[:, 8:10], was[:, 8:10])


def test_rows_of_nobody_and_of_invalid_sequences_stay():
    torch, km = torch_cuda(), _km()
    x = torch.ones((10, 1, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(x, 5.0)
    table = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    # rows 0-1: length below 0; 2-4 fine; 5-8 more than max_rows; 9 nobody's
    seqs = km.KvSeqs(table, torch.tensor([-1, 9, 9], dtype=torch.int32, device="cuda"),
                     torch.tensor([0, 2, 5, 9], dtype=torch.int32, device="cuda"), rows=10, max_rows=3)
    km.kv_rotate(km.kv_rotary(64), seqs, x, q_out=out)
    assert bool((out[[0, 1, 5, 6, 7, 8, 9]] == 5.0).all()) and not bool((out[2:5] == 5.0).any())


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_gradient(layout):
    """The inverse is the adjoint: against the formula's gradient in 64 bits, and against differences (the map is linear, so they
    are exact up to roundings of the results: 2^-22 of their size over the step)."""
    torch, km = torch_cuda(), _km()
    rng = np.random.default_rng(8)
    pos = np.array([3, 70000, 12], np.int32)
    d, dims, amp = 32, 24, 1.5
    x, g = _rows(torch, rng, (3, 2, d), "f32"), _rows(torch, rng, (3, 2, d), "f32")
    rot, at = km.kv_rotary(dims, layout=layout, amplitude=amp), torch.from_numpy(pos).cuda()
    got = km.kv_rotate(rot, at, g, inverse=True)[0].double().cpu()
    xd = x.double().cpu().requires_grad_()
    ang = torch.from_numpy(pos).double()[:, None] * rot.freq.cpu()
    c, s = amp * ang.cos()[:, None], amp * ang.sin()[:, None]
    a, b = (xd[..., :dims // 2], xd[..., dims // 2:dims]) if layout == "halves" else (xd[..., 0:dims:2], xd[..., 1:dims:2])
    u, v = a * c - b * s, a * s + b * c
    y = torch.cat([u, v] if layout == "halves" else [torch.stack([u, v], -1).flatten(-2)], -1)
    (torch.cat([y, xd[..., dims:]], -1) * g.double().cpu()).sum().backward()
    size = g.double().abs().cpu().amax()
    assert (got - xd.grad).abs().max() <= 2 * amp * size * 3 * 2.0 ** -23 + 2.0 ** -24 * 2 * amp * size
    step = 0.5
    for i in range(d):
        e = torch.zeros_like(x)
        e[..., i] = step
        hi, lo = (km.kv_rotate(rot, at, x + sgn * e)[0].double().cpu() for sgn in (1, -1))
        diff = ((hi - lo) / (2 * step) * g.double().cpu()).sum(2)
        room = 2.0 ** -22 * 2 * amp * (x.abs().amax().item() + step) / step * g.abs().sum(2).double().cpu()
        assert ((diff - got[..., i]).abs() <= room).all()


def test_long_calls_and_graph():
    """More rows than a workgroup takes at once, on another stream, captured and replayed with new positions."""
    torch, km = torch_cuda(), _km()
    rng = np.random.default_rng(9)
    x = _rows(torch, rng, (9001, 3, 64), "bf16")
    at = torch.from_numpy(rng.integers(0, 1 << 20, 9001).astype(np.int32)).cuda()
    rot = km.kv_rotary(64)
    freq = 10000.0 ** (-np.arange(32) / 32.0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        out, _ = km.kv_rotate(rot, at, x)
    torch.cuda.synchronize()
    _check(out, x, at.cpu().numpy(), freq, 64, "halves", "bf16")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        held, _ = km.kv_rotate(rot, at, x)
    for i in range(3):
        at += 1000 * i
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, km.kv_rotate(rot, at, x)[0])


def test_not_finite_values_stay_in_their_pair():
    torch, km = torch_cuda(), _km()
    rng = np.random.default_rng(10)
    x = _rows(torch, rng, (4, 2, 64), "bf16")
    at = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    a, _ = km.kv_rotate(km.kv_rotary(64), at, x)
    y = x.clone()
    y[1, 1, 3], y[2, 0, 40] = math.nan, math.inf
    b, _ = km.kv_rotate(km.kv_rotary(64), at, y)
    touched = torch.zeros_like(a, dtype=torch.bool)
    touched[1, 1, [3, 35]] = touched[2, 0, [8, 40]] = True
    assert torch.equal(a[~touched], b[~touched]) and not bool(b[touched].isfinite().any())
