"""Relative position bias, norms of queries and keys with the rotation, stored per-example gradients: the buckets against whole-number
arithmetic, and the arguments that are refused before anything is launched (no GPU needed)."""
import ctypes
import os
import random
import shutil

import pytest

OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, -1, -2, -3, -4
vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_float


@pytest.fixture(scope="module")
def dp():
    from paper_2009_03106_b200 import build as b
    if os.path.exists("/usr/local/cuda/bin/nvcc") or shutil.which("nvcc"):
        b.build()
    elif not os.path.exists(b.LIB):
        pytest.skip("no nvcc and no prebuilt library")
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


def bucket_of(distance, n_buckets, max_distance, bidirectional):
    """floor(m log(d / e) / log(D / e)) is the largest k with d^m e^k >= D^k e^m: no logarithm, no rounding."""
    n, base = n_buckets, 0
    if bidirectional:
        n //= 2
        base, d = (n if distance > 0 else 0), abs(distance)
    else:
        d = max(-distance, 0)
    e = n // 2
    if d < e:
        return base + d
    m, k = n - e, 0
    while k < m - 1 and d ** m * e ** (k + 1) >= max_distance ** (k + 1) * e ** m:
        k += 1
    return base + e + k


@pytest.mark.parametrize("n_buckets,max_distance,bidirectional", [
    (32, 128, True), (32, 128, False), (32, 50, False), (2, 2, False), (3, 9, False), (4, 2, True), (16, 9, False), (64, 4096, True),
    (256, 1 << 24, False), (256, 129, False), (12, 48, False), (7, 81, False)])
def test_buckets_by_whole_numbers(dp, n_buckets, max_distance, bidirectional):
    rng = random.Random(n_buckets * max_distance)
    near = list(range(-300, 301))
    far = [rng.randint(-max_distance - 2, max_distance + 2) for _ in range(100)]
    powers = [s * (n_buckets // 2) * 2 ** k for s in (-1, 1) for k in range(12)] + [s * 3 ** k for s in (-1, 1) for k in range(10)]
    for d in near + far + powers:
        assert dp.dpclip_relbias_bucket(d, n_buckets, max_distance, bidirectional) == bucket_of(d, n_buckets, max_distance, bidirectional), d
    # beyond 32 bits: the last bucket of the direction
    assert dp.dpclip_relbias_bucket(-(1 << 40), n_buckets, max_distance, bidirectional) == (n_buckets // 2 if bidirectional else n_buckets) - 1


def borders_of(n_buckets, max_distance):
    """The smallest distance of every bucket on the logarithmic scale, one direction, by whole numbers."""
    e = n_buckets // 2
    m = n_buckets - e
    for k in range(1, m):
        lo, hi = e, max_distance
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if mid ** m * e ** k >= max_distance ** k * e ** m else (mid + 1, hi)
        yield lo


@pytest.mark.parametrize("n_buckets,max_distance", [
    (100, 2111336), (200, 7419005), (100, 14515163),                # borders a millionth and less above a whole number
    (16, 128), (32, 1024), (16, 1 << 19), (40, 20 << 19), (256, 1 << 24), (255, (1 << 24) - 3), (2, 2), (3, 2)])
def test_both_sides_of_every_border(dp, n_buckets, max_distance):
    for border in borders_of(n_buckets, max_distance):
        for d in (border - 1, border):
            want = bucket_of(-d, n_buckets, max_distance, False)
            assert dp.dpclip_relbias_bucket(-d, n_buckets, max_distance, False) == want, d
            if 2 * n_buckets <= 256:
                assert dp.dpclip_relbias_bucket(-d, 2 * n_buckets, max_distance, True) == want, d
                assert dp.dpclip_relbias_bucket(d, 2 * n_buckets, max_distance, True) == n_buckets + want, d


@pytest.mark.parametrize("n_buckets,max_distance,bidirectional", [(1, 10, False), (0, 10, False), (257, 1000, False), (2, 10, True),
                                                                   (33, 100, True), (32, 8, True), (32, 16, False), (32, (1 << 24) + 1, False)])
def test_bucket_settings_that_are_refused(dp, n_buckets, max_distance, bidirectional):
    with pytest.raises(dp.DpclipError):
        dp.dpclip_relbias_bucket(0, n_buckets, max_distance, bidirectional)


class RelBias(ctypes.Structure):
    _fields_ = [("n_buckets", i32), ("max_distance", i32), ("bidirectional", i32), ("causal", i32)]


class Heads(ctypes.Structure):
    _fields_ = [(n, vp if n in ("x", "dy", "out") else i64) for t in ("x", "dy", "out") for n in (t, t + "_example", t + "_token", t + "_head")] + \
        [("H", i32), ("gain", vp)]


@pytest.fixture(scope="module")
def own(dp):
    return ctypes.CDLL(dp.library_path())           # a handle whose prototypes stay out of the binding's


def at(x):
    return vp(x)


def test_stored_clipped_grad_refusals(own):
    f = own.dpclip_stored_clipped_grad
    f.argtypes = [vp, i64, i32, i32, vp, vp, f32, f32, ctypes.c_ulonglong, ctypes.c_ulonglong, vp]
    good = [at(0x1000), 8, 2, 8, at(0x2000), at(0x3000), 0.0, 1.0, 0, 0, None]
    for pos, value, want in ((0, None, INVALID), (5, None, INVALID), (1, 7, INVALID), (2, 0, INVALID), (3, 0, INVALID), (6, -1.0, INVALID),
                             (6, float("nan"), INVALID), (7, -1.0, INVALID), (0, at(0x1002), MISALIGNED), (4, at(0x2001), MISALIGNED),
                             (5, at(0x3002), MISALIGNED)):
        args = list(good)
        args[pos] = value
        assert f(*args) == want, (pos, value)


def test_relbias_refusals(own):
    c = RelBias(32, 128, 1, 0)
    f = own.dpclip_relbias_forward
    f.argtypes = [vp, i64, ctypes.POINTER(RelBias), i32, i32, i32, i64, i32, vp, i64, i64, vp]
    good = [at(0x1000), 4, ctypes.byref(c), 4, 8, 16, 0, 1, at(0x4000), 16, 128, None]
    for pos, value, want in ((0, None, INVALID), (8, None, INVALID), (2, None, INVALID), (1, 3, INVALID), (3, 0, INVALID), (4, 0, INVALID),
                             (5, -1, INVALID), (6, -1, INVALID), (7, 2, INVALID), (9, 15, INVALID), (10, 127, INVALID), (10, 0, INVALID),
                             (0, at(0x1002), MISALIGNED), (8, at(0x4001), MISALIGNED),
                             (2, ctypes.byref(RelBias(31, 128, 1, 0)), INVALID), (2, ctypes.byref(RelBias(32, 8, 1, 0)), INVALID)):
        args = list(good)
        args[pos] = value
        assert f(*args) == want, (pos, value)
    need = own.dpclip_relbias_workspace_bytes
    need.restype = ctypes.c_size_t
    assert need(2, 4, 8, 16, 32, 1) >= 256 + 2 * 4 * 32 * 4
    g = own.dpclip_relbias_sqnorms
    g.argtypes = [vp, i64, i64, i64, i32, i32, i32, i32, i64, vp, vp, ctypes.POINTER(RelBias), i32, i32, vp, vp, vp, ctypes.c_size_t, vp]
    good = [at(0x1000), 16, 128, 512, 2, 4, 8, 16, 0, None, None, ctypes.byref(c), 1, 0, at(0x5000), at(0x6000), at(0x7000), 1 << 20, None]
    for pos, value, want in ((0, None, INVALID), (14, None, INVALID), (15, None, INVALID), (1, 15, INVALID), (2, -8, INVALID), (3, -8, INVALID),
                             (4, 0, INVALID), (5, 0, INVALID), (6, 0, INVALID), (7, 0, INVALID), (8, -1, INVALID), (11, None, INVALID),
                             (12, 5, INVALID), (0, at(0x1001), MISALIGNED), (9, at(0x1002), MISALIGNED), (10, at(0x1001), MISALIGNED),
                             (14, at(0x5002), MISALIGNED), (15, at(0x6001), MISALIGNED), (16, None, WORKSPACE), (17, 256, WORKSPACE)):
        args = list(good)
        args[pos] = value
        assert g(*args) == want, (pos, value)


def _heads(**other):
    h = Heads(0x1000, 512, 256, 64, 0x2000, 512, 256, 64, 0x3000, 512, 256, 64, 4, 0x4000)
    for n, v in other.items():
        setattr(h, n, v)
    return (Heads * 2)(h, h)


def test_qknorm_refusals(own):
    f = own.dpclip_qknorm_forward
    base = [ctypes.POINTER(Heads), i32, i32, i32, i32, i32, i32, vp, i64, vp, i64, f32, i32]
    f.argtypes = base + [vp]
    good = [_heads(), 2, 2, 2, 64, 64, 0, at(0x8000), 2, None, 0, 1e-6, 1]
    bad = ((0, None, INVALID), (1, 0, INVALID), (1, 3, INVALID), (2, 0, INVALID), (3, 0, INVALID), (4, 0, INVALID), (5, 63, INVALID),
           (5, 66, INVALID), (5, -2, INVALID), (7, None, INVALID), (8, 0, INVALID), (10, -1, INVALID), (11, -1.0, INVALID),
           (11, float("nan"), INVALID), (12, 7, INVALID), (4, 513, UNSUPPORTED), (7, at(0x8002), MISALIGNED), (9, at(0x1001), MISALIGNED),
           (0, _heads(x=None), INVALID), (0, _heads(out=None), INVALID), (0, _heads(H=0), INVALID), (0, _heads(x=0x1001), MISALIGNED),
           (0, _heads(out=0x3001), MISALIGNED), (0, _heads(gain=0x4002), MISALIGNED))
    for pos, value, want in bad:
        args = list(good)
        args[pos] = value
        assert f(*args, None) == want, (pos, value)
    g = own.dpclip_qknorm_backward
    g.argtypes = base + [ctypes.POINTER(vp), ctypes.POINTER(vp), vp, ctypes.c_size_t, vp]
    two = (vp * 2)(0x9000, 0xA000)
    for pos, value, want in bad + ((0, _heads(dy=None), INVALID), (0, _heads(dy=0x2001), MISALIGNED)):
        args = list(good)
        args[pos] = value
        assert g(*args, two, two, at(0xB000), 1 << 20, None) == want, (pos, value)
    assert g(*good, None, two, at(0xB000), 1 << 20, None) == INVALID
    assert g(*good, two, None, at(0xB000), 1 << 20, None) == INVALID
    assert g(*good, (vp * 2)(0x9002, 0xA000), two, at(0xB000), 1 << 20, None) == MISALIGNED
    assert g(*good, two, two, None, 0, None) == WORKSPACE
    assert g(*good, two, two, at(0xB000), 300, None) == WORKSPACE
    need = own.dpclip_qknorm_workspace_bytes
    need.restype = ctypes.c_size_t
    assert need(2, 2, 4, 4, 64) >= 256 + 2 * 2 * 64 * 4
    r = own.dpclip_rotation_table
    r.argtypes = [vp, i64, i32, ctypes.c_double, ctypes.c_double, vp]
    for args in ((None, 4, 8, 1e4, 1.0), (at(0x10), 0, 8, 1e4, 1.0), (at(0x10), 4, 7, 1e4, 1.0), (at(0x10), 4, 0, 1e4, 1.0),
                 (at(0x10), 4, 8, 0.0, 1.0), (at(0x10), 4, 8, 1e4, 0.0)):
        assert r(*args, None) == INVALID, args


def test_gated_refusals(own):
    f, b = own.dpclip_gated_forward, own.dpclip_gated_backward
    f.argtypes = [vp, i64, vp, i64, vp, i32, i32, i32, i32, i32, vp, i64, vp, i64, vp, ctypes.c_size_t, vp]
    good = [at(0x1000), 64, at(0x2000), 64, at(0x3000), 16, 64, 32, 1, 0, at(0x4000), 32, at(0x5000), 64, at(0x10000), 1 << 30, None]
    for pos, value, want in ((0, None, INVALID), (2, None, INVALID), (10, None, INVALID), (1, 63, INVALID), (3, 63, INVALID), (11, 31, INVALID),
                             (13, 63, INVALID), (5, 0, INVALID), (6, 0, INVALID), (7, 0, INVALID), (8, 2, INVALID), (9, 4, INVALID), (9, -1, INVALID),
                             (0, at(0x1001), MISALIGNED), (2, at(0x2001), MISALIGNED), (4, at(0x3002), MISALIGNED), (10, at(0x4001), MISALIGNED),
                             (12, at(0x5001), MISALIGNED), (14, None, WORKSPACE), (14, at(0x10010), WORKSPACE), (15, 255, WORKSPACE)):
        args = list(good)
        args[pos] = value
        assert f(*args) == want, (pos, value)
    b.argtypes = [vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, i32, vp, i64, vp, i64, vp, ctypes.c_size_t, vp]
    good = [at(0x1000), 32, at(0x2000), 64, at(0x3000), 64, 16, 64, 32, 1, 0, at(0x4000), 64, at(0x5000), 64, at(0x10000), 1 << 30, None]
    for pos, value, want in ((0, None, INVALID), (2, None, INVALID), (4, None, INVALID), (11, None, INVALID), (1, 31, INVALID), (3, 63, INVALID),
                             (5, 63, INVALID), (12, 63, INVALID), (14, 63, INVALID), (6, 0, INVALID), (7, 0, INVALID), (8, 0, INVALID), (9, 7, INVALID),
                             (10, 9, INVALID), (0, at(0x1001), MISALIGNED), (2, at(0x2001), MISALIGNED), (4, at(0x3001), MISALIGNED),
                             (11, at(0x4001), MISALIGNED), (13, at(0x5001), MISALIGNED), (15, None, WORKSPACE), (16, 255, WORKSPACE)):
        args = list(good)
        args[pos] = value
        assert b(*args) == want, (pos, value)


def test_host_tensors_are_refused(dp):
    """The library reads device memory: a tensor of the host never reaches it."""
    import torch
    x = torch.zeros(2, 3, 4, 8)
    with pytest.raises(ValueError):
        dp.dpclip_qknorm_forward(x, None, None, None, None, x, None)
    with pytest.raises(ValueError):
        dp.dpclip_relbias_forward(torch.zeros(32, 4), torch.zeros(4, 2, 2), 128)
    with pytest.raises(ValueError):
        dp.dpclip_stored_clipped_grad(torch.zeros(2, 4), None, torch.zeros(4))


def test_expanded_workspaces_are_refused(dp):
    """An expanded tensor counts bytes that it does not own; the refusal comes before anything about devices."""
    import torch
    ws = torch.zeros((1,), dtype=torch.uint8).expand(1 << 24)
    t = lambda *s: torch.zeros(s)                                             # noqa: E731
    calls = [
        lambda: dp.dpclip_relbias_sqnorms(t(1, 1, 4, 4), t(1, 8, 1), t(1), ws, 64),
        lambda: dp.dpclip_qknorm_backward(t(1, 4, 1, 8), None, t(1, 4, 1, 8), None, t(8), None, None, t(1, 4, 1, 8), None, t(1, 8), None, t(1), None, ws),
        lambda: dp.dpclip_gated_forward(t(4, 8), t(16, 8), None, t(4, 8), None, dp.DPCLIP_ACT_SILU, ws),
    ]
    for call in calls:
        with pytest.raises(ValueError, match="workspace"):
            call()
