"""What the host refuses of rotary positions, rotated appends, the 4-bit cache and sampling (no GPU needed: every check comes before a launch)."""
import ctypes as C
import math

import pytest
import torch

from paper_2604_07853_amd import binding as q

PTR = 4096      # an aligned address that is never followed


@pytest.fixture(scope="module")
def L():
    return q.lib()


@pytest.fixture(scope="module")
def rope(L):
    return q.Rope(64)


def text(L):
    return L.qarl_last_error().decode()


def test_frequencies(L):
    f, a = q.qarl_rope_frequencies(64, 10000.0)
    assert a == 1.0 and all(abs(x - 10000.0 ** (-2 * i / 64)) <= 1e-15 for i, x in enumerate(f))
    g, _ = q.qarl_rope_frequencies(64, 10000.0, q.QARL_ROPE_LINEAR, 4.0)
    assert all(abs(x - y / 4) <= 1e-16 for x, y in zip(g, f))
    y, a = q.qarl_rope_frequencies(64, 10000.0, q.QARL_ROPE_YARN, 8.0, 4096, 1.0, 32.0)
    assert abs(a - (0.1 * math.log(8.0) + 1)) < 1e-7
    turns = [4096 * x / (2 * math.pi) for x in f]
    for i in range(32):         # the ends: pairs of many turns as they are, of few stretched, in between falling
        if turns[i] > 45:
            assert y[i] == f[i]
        if turns[i] < 0.7:
            assert abs(y[i] - f[i] / 8) < 1e-18
        assert f[i] / 8 * (1 - 1e-12) <= y[i] <= f[i]
    b, a = q.qarl_rope_frequencies(64, 10000.0, q.QARL_ROPE_BANDS, 8.0, 4096, 1.0, 4.0)
    assert a == 1.0
    for i in range(32):
        keep = min(max((turns[i] - 1) / 3, 0), 1)
        assert abs(b[i] - (f[i] * keep + f[i] / 8 * (1 - keep))) <= 1e-15


def test_frequency_refusals(L):
    f, a = (C.c_double * 64)(), C.c_float()
    good = [64, 1e4, q.QARL_ROPE_YARN, 8.0, 4096.0, 1.0, 32.0]
    for at, value in ((0, 0), (0, 24), (0, 272), (1, 1.0), (1, math.nan), (1, math.inf), (2, 7), (3, 0.5), (3, math.nan), (4, 0.0), (5, 0.0), (5, 40.0), (6, math.inf)):
        args = list(good)
        args[at] = value
        assert L.qarl_rope_frequencies(*args, f, C.byref(a)) in (q.QARL_ERR_INVALID_ARG, q.QARL_ERR_UNSUPPORTED), (at, value)
    assert L.qarl_rope_frequencies(*good, None, C.byref(a)) == q.QARL_ERR_INVALID_ARG
    assert L.qarl_rope_frequencies(*good, f, C.byref(a)) == 0
    for kw in (dict(frequencies=[0.1] * 31), dict(frequencies=[4.0] * 32), dict(frequencies=[math.nan] * 32), dict(amplitude=0.0), dict(amplitude=math.inf), dict(layout=2)):
        with pytest.raises((ValueError, q.QarlError)):
            q.Rope(64, **kw)


def test_rotary_refusals(L, rope):
    good = dict(rope=rope.ref, positions=PTR, T=3, D=64, dtype=0, q=PTR, qt=256, qh=64, heads=4, qo=PTR, qot=256, qoh=64, k=PTR, kt=128, kh=64, kheads=2, ko=PTR, kot=128,
                koh=64)

    def status(**kw):
        return L.qarl_rotary(*dict(good, **kw).values(), 0, None)
    for kw, rc in ((dict(rope=None), -1), (dict(rope=C.byref(q.qarl_rope())), -1), (dict(positions=None), -1), (dict(T=-1), -1), (dict(D=72), -2), (dict(D=48), -1),
                   (dict(D=2048), -2), (dict(dtype=3), -1), (dict(q=None), -1), (dict(qo=None), -1), (dict(q=PTR + 8), -3), (dict(qt=260), -3), (dict(qh=60), -3),
                   (dict(heads=-1), -1), (dict(qot=192), -1), (dict(qoh=32, qot=1024), -1), (dict(qot=0), -1), (dict(positions=PTR + 4), -3), (dict(k=None), -1),
                   (dict(kot=64), -1)):
        assert status(**kw) == rc, (kw, text(L))
        assert "qarl_rotary" in text(L)
    assert status(T=0) == 0 and status(heads=0, kheads=0) == 0
    assert status(T=0, q=None, k=None, positions=None) == 0


def cache_desc(fmt, **kw):
    d = dict(fmt=fmt, num_pages=4, page_size=16, kv_heads=2, head_dim=64, k=PTR, v=PTR, k_scales=PTR, v_scales=PTR)
    d.update(kw)
    return C.byref(q.qarl_kv_cache(*d.values()))


def test_append_and_cache_refusals(L, rope):
    good = dict(cache=cache_desc(3), rope=rope.ref, positions=PTR, T=3, q=PTR, qt=256, qh=64, heads=4, qo=PTR, qot=256, qoh=64, k=PTR, kt=128, kh=64, v=PTR, vt=128, vh=64,
                slots=PTR)

    def status(**kw):
        return L.qarl_rotary_kv_write(*dict(good, **kw).values(), None)
    for kw, rc in ((dict(cache=None), -1), (dict(cache=cache_desc(4)), -2), (dict(cache=cache_desc(3, k_scales=None)), -1), (dict(cache=cache_desc(3, v_scales=PTR + 4)), -3),
                   (dict(cache=cache_desc(3, head_dim=96)), -2), (dict(rope=None), -1), (dict(rope=q.Rope(128).ref), -1), (dict(positions=None), -1), (dict(T=-1), -1),
                   (dict(heads=-1), -1), (dict(q=None), -1), (dict(qo=None), -1), (dict(qot=128), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(slots=None), -1),
                   (dict(kt=4), -3), (dict(vh=4), -3), (dict(k=PTR + 2), -3), (dict(slots=PTR + 4), -3)):
        assert status(**kw) == rc, (kw, text(L))
    assert status(T=0) == 0
    assert L.qarl_kv_cache_bytes(q.QARL_KV_E2M1, 3, 16, 2, 128) == 3 * 16 * 2 * 64 and L.qarl_kv_scales_bytes(q.QARL_KV_E2M1, 3, 16, 2, 128) == 3 * 16 * 2 * 4
    assert L.qarl_kv_cache_bytes(4, 3, 16, 2, 128) == 0


def test_sample_refusals(L):
    good = dict(logits=PTR, dtype=0, stride=100, T=3, V=100, u=PTR, temperature=PTR, top_k=PTR, top_p=PTR, min_p=PTR, token=PTR, logprob=PTR, kept=PTR, ws=PTR, bytes=1 << 40)

    def status(**kw):
        return L.qarl_sample(*dict(good, **kw).values(), None)
    for kw, rc in ((dict(logits=None), -1), (dict(u=None), -1), (dict(token=None), -1), (dict(T=-1), -1), (dict(V=0), -1), (dict(V=(1 << 20) + 1, stride=1 << 21), -2),
                   (dict(stride=99), -1), (dict(dtype=2), -1), (dict(logits=PTR + 1), -3), (dict(dtype=1, logits=PTR + 2), -3), (dict(u=PTR + 2), -3), (dict(top_k=PTR + 1), -3),
                   (dict(token=PTR + 2), -3)):
        assert status(**kw) == rc, (kw, text(L))
    if L.qarl_sample_workspace_bytes(3, 100):
        assert status(ws=None) == -4 and status(bytes=L.qarl_sample_workspace_bytes(3, 100) - 1) == -4 and status(ws=PTR + 4) == -4
    assert status(T=0) == 0 and L.qarl_sample_workspace_bytes(0, 100) == 0


def test_the_binding_refuses_what_is_not_on_the_gpu_or_of_another_shape(rope):
    x, pos = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="q must be"):
        q.qarl_rotary(rope, pos, x)
    with pytest.raises(ValueError, match="q must be"):
        q.qarl_rotary(rope, pos, x[0])
    with pytest.raises(ValueError, match="without k"):
        q.qarl_rotary(rope, pos, x, k_out=x)
    with pytest.raises(ValueError):
        q.qarl_rotary_kv_write(q.KVCache.empty(q.QARL_KV_E2M1, 2, 16, 4, 64, "cpu"), rope, pos, x, x, x, pos)
    with pytest.raises(ValueError, match="logits must be"):
        q.qarl_sample(torch.zeros((2, 10)), torch.zeros(2))
    c = q.KVCache.empty(q.QARL_KV_E2M1, 2, 16, 4, 64, "cpu")
    assert c.head_dim == 64 and c.k.shape == (2, 4, 16, 32) and c.k_scales.shape == (2, 4, 16, 4)
    for bad in ((c.k, c.v), (c.k, c.v, c.k_scales, c.v_scales.float()), (c.k, c.v, c.k_scales[..., :2], c.v_scales), (c.k.to(torch.bfloat16), c.v, c.k_scales, c.v_scales)):
        with pytest.raises(ValueError):
            q.KVCache(q.QARL_KV_E2M1, *bad)
    with pytest.raises(ValueError, match="even"):
        q.KVCache.empty(q.QARL_KV_E2M1, 2, 16, 4, 63, "cpu")


@pytest.mark.parametrize("base,length,low,high", [(1e4, 4.0, 1.0, 32.0), (1e4, 1.0, 1.0, 32.0), (1e4, 6.25, 1.0, 32.0), (1e4, 40.0, 8.0, 32.0), (1e4, 200.0, 1.0, 32.0), (5.0, 300.0, 1.0, 2.0),
                                                  (1e6, 1e17, 1.0, 32.0)])
def test_stretched_frequencies_at_the_ends(L, base, length, low, high):
    """Pairs of fewer than `low` turns are stretched and those of more than `high` are not, also where that is all pairs, the first among them."""
    f, _ = q.qarl_rope_frequencies(64, base)
    y, _ = q.qarl_rope_frequencies(64, base, q.QARL_ROPE_YARN, 8.0, length, low, high)
    for i in range(32):
        turns = length * f[i] / (2 * math.pi)
        if turns > high * (1 + 1e-9):
            assert y[i] == f[i], i
        elif turns < low * (1 - 1e-9):
            assert abs(y[i] - f[i] / 8) <= 1e-15 * f[i], i
        assert f[i] / 8 * (1 - 1e-12) <= y[i] <= f[i] * (1 + 1e-12), i
