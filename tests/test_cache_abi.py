"""The 8-bit key/value cache without a GPU: its oracle against hand arithmetic, and what the C entry points and the binding refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_19835_amd import binding as rb


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(rb.LIB_PATH):
        from paper_2511_19835_amd.build import build_library
        build_library(verbose=False)
    return rb.load_library()


# ---- the oracle ----------------------------------------------------------------------------------
def test_rounding_to_e4m3_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 40001), np.ldexp(np.linspace(-16, 16, 4097), -9), [0.0, -0.0]])
    x = torch.from_numpy(x).float()
    want = x.to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(co.round_e4m3(x.double().numpy()), want)
    assert np.isnan(co.round_e4m3(np.array([np.inf, -np.inf, np.nan]))).all()


@pytest.mark.parametrize("amax,largest,least,e", [(448, 448, -126, 0), (449, 448, -126, 1), (224, 448, -126, -1), (225, 448, -126, 0),
                                                  (0, 448, -126, -126), (1e-45, 448, -126, -126), (127, 127, -100, 0), (128, 127, -100, 1),
                                                  (2.0 ** 127 * 1.75, 448, -126, 119), (2.0 ** 127 * 1.9, 448, -126, 120)])
def test_least_exponent(amax, largest, least, e):
    assert co.least_exponent(amax, largest, least) == e


def test_oracle_token_by_token_is_the_same_as_at_once():
    rng = np.random.default_rng(0)
    K, V = rng.normal(size=(2, 1, 1, 100, 64))
    at_once, by_token = (co.Cache(1, 64, 64, [[1, 0]], 2) for _ in range(2))
    at_once.write(K, V, [0])
    for t in range(100):
        by_token.write(K[:, :, t:t + 1], V[:, :, t:t + 1], [t])
    for key, p in at_once.held.items():
        q = by_token.held[key]
        assert (p.ek, p.ev, p.em) == (q.ek, q.ev, q.em)
        # rounded twice: half a step of the smallest values each time
        np.testing.assert_allclose(p.k, q.k, rtol=0, atol=2.0 ** (p.ek - 9))
    O = at_once.attend(K[:, :, -1:], [100], None, 0.0, True)
    k, v, there = at_once.rows(0, 0, 0, 100)
    assert there.all()
    s = k @ K[0, 0, -1] / 8
    np.testing.assert_allclose(O["O"][0, 0, 0], np.exp(s - s.max()) @ v / np.exp(s - s.max()).sum(), rtol=1e-12)


@pytest.mark.parametrize("by", [20, 40, 100])
def test_the_bound_of_a_row_is_made_of_its_own_keys(by):
    """Zeros in place of the outputs are outside the bound of the attention's tests, also beside blocks of much larger values that the row
    is not to read or gives no weight to."""
    rng = np.random.default_rng(0)
    c = co.Cache(1, 64, 64, [range(8)], 8)
    K = rng.normal(size=(1, 1, 512, 64)) * 0.1
    V = rng.normal(size=K.shape) * np.repeat(2.0 ** np.array([0, -by, 3, by, -2, by // 2, -by // 2, 1]), 64).reshape(1, 1, 512, 1)
    K[0, 0, 3 * 64:4 * 64, 0] = -60.0                      # no weight on the block of the largest values
    c.write(K, V, [0])
    Q = rng.normal(size=(1, 1, 3, 64)) * 0.1
    Q[..., 0] = 100.0
    for own in ([1], [1, 6], [2, 3, 7]):
        r = c.attend(Q, [512], None, 0.0, False, {(0, 0, 0): own}, 3)
        es = (64 + 16) * 2.0 ** -24 * r["S"]
        bound = 2.0 ** -8 * np.abs(r["O"]) + (2.0 ** -11 + 2 * es + 4 * r["n"] * 2.0 ** -24)[..., None] * r["A"] + (r["n"] * 2.0 ** -24 * r["vmax"])[..., None]
        assert ((np.abs(r["O"]) > bound).mean(-1) > 0.9).all()


# ---- refusals ------------------------------------------------------------------------------------
ONE = 256                         # an address that is never read: validation fails first


def _cache(**kw):
    base = dict(batch=2, heads_kv=2, head_dim=128, block=64, max_blocks=10, pages=20, k_codes=ONE, v_codes=ONE, scales=ONE, k_mean=ONE, table=ONE)
    base.update(kw)
    return rb.rsa_cache(**base)


def _rows(heads=2, t=5, sb=5 * 2 * 128, sh=5 * 128, st=128):
    return rb.rsa_rows(heads, t, sb, sh, st)


BAD_CACHES = [(dict(batch=0), -2), (dict(heads_kv=0), -2), (dict(max_blocks=0), -2), (dict(pages=0), -2), (dict(head_dim=96), -3),
              (dict(block=32), -3), (dict(batch=40000), -3), (dict(pages=1 << 31), -3), (dict(max_blocks=1 << 26), -3)]


@pytest.mark.parametrize("kw,code", BAD_CACHES + [(dict(k_codes=None), -1), (dict(v_codes=None), -1), (dict(scales=None), -1), (dict(k_mean=None), -1),
                                                  (dict(table=None), -1), (dict(k_codes=264), -2), (dict(scales=260), -2), (dict(table=258), -2)])
def test_bad_caches_are_refused(lib, kw, code):
    c, r, R = _cache(**kw), _rows(), _rows(heads=4, sb=5 * 4 * 128)
    by = ctypes.byref
    assert lib.rsa_cache_write(by(c), by(r), ONE, ONE, ONE, None, None) == code
    assert lib.rsa_cache_read(by(c), by(r), ONE, None, ONE, 512, None) == code
    assert lib.rsa_cache_select(by(c), by(R), ONE, ONE, None, 1, 1, 0, 0, 0, ONE, ONE, 10, None, 0, None) == code
    assert lib.rsa_cache_attn(by(c), by(R), ONE, ONE, None, 0.0, 0, None, None, 0, 0, ONE, None, None, 0, None) == code


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_sizes_of_bad_caches_are_refused(lib, kw, code):
    c = _cache(k_codes=None, v_codes=None, scales=None, k_mean=None, table=None, **kw)
    n = ctypes.c_size_t()
    assert lib.rsa_cache_bytes(ctypes.byref(c), n, n, n) == code


def test_sizes(lib):
    c = _cache(k_codes=None, v_codes=None, scales=None, k_mean=None, table=None)
    assert rb.rsa_cache_bytes(c) == (20 * 2 * 64 * 128, 20 * 2 * 16, 20 * 2 * 128)
    assert lib.rsa_cache_bytes(None, None, None, None) == -1
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.rsa_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(_rows(heads=4)), 0, a, b) == 0 and (a.value, b.value) == (0, 0)   # ten blocks: one launch
    long = _cache(max_blocks=5000, k_codes=None, v_codes=None, scales=None, k_mean=None, table=None)
    assert lib.rsa_cache_workspace_bytes(ctypes.byref(long), ctypes.byref(_rows(heads=4)), 1, a, b) == 0 and a.value == 2 * 2 * 5 * 5000 * 4 and b.value > 0
    assert lib.rsa_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(_rows(heads=4)), -1, a, b) == -5
    assert lib.rsa_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(_rows(heads=3)), 0, a, b) == -2


@pytest.mark.parametrize("rows,code", [(None, -1), (dict(heads=0), -2), (dict(t=0), -2), (dict(st=64), -2), (dict(st=132), -2), (dict(sb=0), -2),
                                       (dict(sh=4), -2), (dict(heads=3), -2), (dict(t=1 << 28), -3)])
def test_bad_rows_are_refused(lib, rows, code):
    c, by = _cache(), ctypes.byref
    r = None if rows is None else by(_rows(**rows))
    assert lib.rsa_cache_attn(by(c), r, ONE, ONE, None, 0.0, 0, None, None, 0, 0, ONE, None, None, 0, None) == code
    assert lib.rsa_cache_select(by(c), r, ONE, ONE, None, 1, 1, 0, 0, 0, ONE, ONE, 10, None, 0, None) == code
    assert lib.rsa_cache_write(by(c), r, ONE, ONE, ONE, None, None) == code


def test_bad_arguments_are_refused(lib):
    c, r, R, by = _cache(), _rows(), _rows(heads=4), ctypes.byref
    write = lambda K=ONE, V=ONE, start=ONE, rows=r: lib.rsa_cache_write(by(c), by(rows), K, V, start, None, None)
    assert write(K=None) == -1 and write(V=None) == -1 and write(start=None) == -1 and write(K=264) == -2 and write(rows=R) == -2
    read = lambda K=ONE, V=512, start=ONE: lib.rsa_cache_read(by(c), by(r), start, None, K, V, None)
    assert read(K=None) == -1 and read(V=264) == -2 and read(V=ONE) == -5 and read(start=None) == -1

    def select(Q=ONE, kv=ONE, group=1, keep=4, first=1, last=1, flags=0, idx=ONE, kept=ONE, n=10, ws=None, cache=c):
        return lib.rsa_cache_select(by(cache), by(R), Q, kv, None, group, keep, first, last, flags, idx, kept, n, ws, 0, None)
    assert select(Q=None) == -1 and select(kv=None) == -1 and select(idx=None) == -1 and select(kept=None) == -1 and select(Q=264) == -2
    assert select(group=0) == -5 and select(keep=0) == -5 and select(first=-1) == -5 and select(last=-1) == -5 and select(flags=2) == -5
    assert select(n=0) == -5 and select(n=3) == -5 and select(keep=9, n=8) == -5 and select(group=128, n=4) == -5 and select(last=2**31 - 1, n=9) == -5
    assert select(ws=8) == -4
    assert select(cache=_cache(max_blocks=16385), n=16385) == -3

    def attn(Q=ONE, kv=ONE, scale=0.0, flags=0, idx=None, kept=None, group=0, n=0, O=ONE, ws=None, nws=0, cache=c):
        return lib.rsa_cache_attn(by(cache), by(R), Q, kv, None, scale, flags, idx, kept, group, n, O, None, ws, nws, None)
    assert attn(Q=None) == -1 and attn(kv=None) == -1 and attn(O=None) == -1 and attn(idx=ONE) == -1 and attn(kept=ONE) == -1
    assert attn(Q=264) == -2 and attn(O=264) == -2 and attn(scale=-1.0) == -5 and attn(scale=math.nan) == -5 and attn(scale=math.inf) == -5
    assert attn(flags=2) == -5 and attn(idx=ONE, kept=ONE, group=0, n=4) == -5 and attn(idx=ONE, kept=ONE, group=1, n=0) == -5
    # more workgroups than a launch takes: refused by the host
    many = _rows(heads=4, t=1 << 23, sb=(1 << 23) * 4 * 128, sh=(1 << 23) * 128)
    assert lib.rsa_cache_attn(by(c), by(many), ONE, ONE, None, 0.0, 0, ONE, ONE, 1, 4, ONE, None, None, 0, None) == -3
    assert lib.rsa_cache_select(by(c), by(many), ONE, ONE, None, 1, 4, 1, 1, 0, ONE, ONE, 10, None, 0, None) == -3
    assert attn(ws=ONE, nws=16, cache=_cache(max_blocks=100)) == -4 and attn(ws=264, nws=1 << 30) == -4
    assert select(ws=ONE, cache=_cache(max_blocks=5000), n=10) == -4                     # scores need a workspace there


def test_binding_refuses_cpu_tensors_and_wrong_buffers(lib):
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    args = dict(k_codes=u8(4, 2, 64 * 64), v_codes=u8(4, 2, 64 * 64), scales=torch.zeros(4, 2, 4), k_mean=torch.zeros(4, 2, 64, dtype=torch.int8),
                table=torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="device tensors only"):
        rb.cache_of(**args, block=64)
    for name, bad in (("v_codes", u8(4, 2, 64 * 32)), ("scales", torch.zeros(4, 2, 2)), ("k_mean", torch.zeros(4, 2, 64)),
                      ("table", torch.zeros(1, 4)), ("scales", torch.zeros(4, 4, 2).transpose(1, 2))):
        with pytest.raises(ValueError):
            rb.cache_of(**{**args, name: bad}, block=64)
    with pytest.raises(AssertionError):
        rb.make_rows(torch.zeros(1, 2, 3, 64))
    r = rb.make_rows(torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16).transpose(1, 2))
    assert (r.heads, r.t, r.stride_h, r.stride_t) == (2, 3, 64, 128)


def test_binding_refuses_a_workspace_elsewhere(lib):
    """On another device than the cache, or a view that says more bytes than it has."""
    on = lambda device: type("Tensor", (), dict(device=torch.device(device), is_cuda=True, is_contiguous=lambda self: True, stride=lambda self: (1,),
                                                numel=lambda self: 1024, element_size=lambda self: 1, data_ptr=lambda self: 256))()
    cache = type("Cache", (), dict(device=torch.device("cuda:0")))()
    assert rb._scratch(cache, on("cuda:0")) == (256, 1024) and rb._scratch(cache, None) == (None, 0)
    with pytest.raises(ValueError, match="workspace"):
        rb._scratch(cache, on("cuda:1"))
    with pytest.raises(ValueError, match="workspace"):
        rb._scratch(cache, torch.zeros(1024, dtype=torch.uint8))
    cache.device = torch.device("cpu")
    with pytest.raises(ValueError, match="workspace"):
        rb._scratch(cache, torch.zeros(1, dtype=torch.uint8).expand(1 << 20))


@pytest.mark.parametrize("scale", [3e38, 2.4e38, -1e-45, math.inf, -math.inf, math.nan])
def test_scales_beyond_32_bits_are_refused(lib, scale):
    """Scores are powers of two inside: 2.4e38 * log2(e) is none that fp32 holds."""
    by = ctypes.byref
    assert lib.rsa_cache_attn(by(_cache()), by(_rows(heads=4)), ONE, ONE, None, scale, 0, None, None, 0, 0, ONE, None, None, 0, None) == -5
