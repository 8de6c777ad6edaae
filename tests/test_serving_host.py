"""CPU: the host side of the cache, attention and sampling entry points, and
the oracle's definitions of them."""
import ctypes

import numpy as np
import pytest

import oracle as O


def test_cache_geometry(sdq):
    assert sdq.sdq_cache_bytes(sdq.CacheDesc(8, 128, 16, 10)) == 10 * 8 * 16 * 128 * 2
    for bad in (sdq.CacheDesc(0, 128, 16, 1), sdq.CacheDesc(8, 80, 16, 1), sdq.CacheDesc(8, 128, 8, 1), sdq.CacheDesc(8, 128, 256, 1),
                sdq.CacheDesc(8, 128, 16, -1), sdq.CacheDesc(1 << 10, 64, 128, 1 << 14)):
        assert sdq.sdq_cache_bytes(bad) == 0


def test_null_handles_are_refused(sdq):
    L = sdq.lib()
    assert L.sdq_cache_create(None, None, None, None) == -1
    h = ctypes.c_void_p()
    assert L.sdq_cache_create(ctypes.byref(sdq.CacheDesc(8, 128, 16, 1).c()), None, None, ctypes.byref(h)) == -1
    assert L.sdq_cache_destroy(None) == -1
    assert L.sdq_cache_append(None, None, 1, None, 0, None, 0, None, 0, 0, None, None, None) == -1


def test_rope_table(sdq):
    cos, sin = sdq.sdq_rope_table(5000, 64, 10000.0)
    p, j = np.meshgrid(np.arange(5000), np.arange(32), indexing="ij")
    a = p * 10000.0 ** (-j / 32)
    # fp64 angles differ by their own rounding (2^-52 of up to 5000), the tables by one rounding to fp32
    assert np.abs(cos - np.cos(a)).max() <= 2.0 ** -25 + 2.0 ** -38 and np.abs(sin - np.sin(a)).max() <= 2.0 ** -25 + 2.0 ** -38
    for bad in ((0, 64, 1e4), (4, 7, 1e4), (4, 0, 1e4), (4, 8, 0.0), (4, 8, float("inf"))):
        with pytest.raises(sdq.SdqError):
            sdq.sdq_rope_table(*bad)


def test_oracle_rotation_is_a_rotation_by_position():
    """Scores of rotated queries and keys depend on the distance of their positions alone; pairs keep their length."""
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 16))
    a = np.arange(200)[:, None] * 100.0 ** (-np.arange(6) / 6)
    cos, sin = np.cos(a), np.sin(a)
    for inter in (False, True):
        d = [O.serving.rotate(q, p + 7, cos, sin, inter) @ O.serving.rotate(k, p, cos, sin, inter).T for p in (0, 40, 190)]
        assert np.ptp(d) < 1e-12
        r = O.serving.rotate(q, 33, cos, sin, inter)
        assert np.array_equal(r[:, 12:], q[:, 12:]) and abs(np.linalg.norm(r) - np.linalg.norm(q)) < 1e-12


def test_oracle_append_and_attend_by_hand():
    """Two tokens of one sequence behind a prefix of one: the first sees two keys, the second three."""
    kp, vp = np.zeros((3, 1, 2, 2)), np.zeros((3, 1, 2, 2))
    kp[2, 0, 0], vp[2, 0, 0] = [0, 0], [8, 0]                       # the prefix, on page 2
    cos, sin = np.ones((9, 1)), np.zeros((9, 1))
    q = np.array([[[1.0, 0]], [[1.0, 0]]])
    new = np.array([[[np.log(3), 5.0]], [[np.log(4), -5.0]]])
    v = np.array([[[0, 4.0]], [[16.0, 0]]])
    _, kp, vp = O.serving.append(q, new, v, kp, vp, [0, 2], [2], [[1]], 1, cos, sin, False)
    assert np.array_equal(kp[1, 0], new[:, 0])
    out, lse, _ = O.serving.attend(q, kp, vp, [0, 2], [2], [[1]], [2], 1, 1.0)
    assert np.allclose(out[0, 0], [8 / 4, 4 * 3 / 4]) and np.allclose(out[1, 0], [(8 + 64) / 8, 12 / 8])
    assert np.allclose(lse[:, 0], np.log([4, 8]))
    out, lse, _ = O.serving.attend(q[:1], kp, vp, [0, 1], [0], [[1]], [], 0, 1.0)
    assert np.all(out == 0) and np.all(lse == -np.inf)


def test_oracle_sampling_by_hand():
    """Weights 8 : 4 : 2 : 1 : 1 at indices 3, 0, 4, 1, 2."""
    z = np.log([4.0, 1.0, 1.0, 8.0, 2.0])
    pick = lambda u, *a: O.serving.sample_row(z, u, *a)[0]
    assert [pick(u) for u in (0.0, 0.24, 0.26, 0.32, 0.4, 0.8, 0.95)] == [0, 0, 1, 2, 3, 3, 4]
    assert pick(0.9, 0.0) == 3 and pick(0.9, 1.0, 1) == 3
    assert [pick(u, 1.0, 2) for u in (0.3, 0.4)] == [0, 3]
    assert [pick(u, 1.0, 4) for u in (0.28, 0.9)] == [1, 4]                     # index 2 ties with 1 and is out
    assert [pick(u, 1.0, 0, 0.7) for u in (0.3, 0.34)] == [0, 3]                # 8 of 16 lie before index 0, 12 before 4
    assert [pick(u, 1.0, 0, 1.0, 0.2) for u in (0.28, 0.3, 0.9)] == [0, 3, 4]
    assert [pick(u, 0.5, 3) for u in (0.15, 0.25, 0.97)] == [0, 3, 4]           # squares: 64 : 16 : 4
    assert O.serving.sample_row([-np.inf, np.nan], 0.5)[0] == -1


def test_sample_null_pointers_are_refused(sdq):
    assert sdq.lib().sdq_sample(None, 0, 1, 10, 10, None, None, None, None, None, None, None) == -1
    assert sdq.lib().sdq_attention(None, None, 1, None, 0, 1.0, None, None, None, 0, None) == -1
    assert sdq.lib().sdq_attention_workspace_bytes(None, None, 1) == 0
