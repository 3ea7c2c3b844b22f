"""The 4-bit cache, page assignment and rotary positions without a GPU: their oracle against hand arithmetic, and what the C entry points and
the binding refuse."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import serve_oracle as so
from paper_2511_19835_amd import binding as rb


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(rb.LIB_PATH):
        from paper_2511_19835_amd.build import build_library
        build_library(verbose=False)
    return rb.load_library()


# ---- the oracle ----------------------------------------------------------------------------------
def test_rounding_to_e2m1():
    x = np.array([0.0, 0.24, 0.25, 0.26, 0.74, 0.75, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 4.99, 5.0, 5.01, 6.0, -0.75, -5.0])
    np.testing.assert_array_equal(so.round_e2m1(x), [0, 0, 0, 0.5, 0.5, 1, 1, 1.5, 2, 2, 3, 4, 4, 4, 6, 6, -1, -4])
    y = np.linspace(-6, 6, 4001)
    assert (np.abs(so.round_e2m1(y) - y) <= np.abs(y[:, None] - np.concatenate([so.LEVELS, -so.LEVELS])).min(1) + 1e-15).all()


def test_what_a_row_holds():
    x = np.zeros(64)
    x[:32], x[32:] = 6.0, np.linspace(0, 2.0 ** -30, 32)
    s = so.stored(x, 32)
    assert (s[:32] == 6).all() and s[63] == 2.0 ** -30 and np.abs(s[32:] - x[32:]).max() <= 2.0 ** -32 * (1 + 1e-12)   # e = -32; steps of 2 e at the top, half of that
    assert so.stored(np.full(32, 6.0625), 32)[0] == 6.0                        # e = 1: 3.03 is 3
    x[40] = np.nan
    s = so.stored(x, 32)
    assert (s[:32] == 6).all() and np.isnan(s[32:]).all()
    assert np.isnan(so.stored(x, 64)).all()
    assert np.isposinf(so.stored(np.full(32, 1.75 * 2.0 ** 127), 32)).all()
    assert (so.stored(np.full(32, 2.0 ** -127), 32) == 0).all() and so.stored(np.full(32, 2.0 ** -125), 32)[0] == 2.0 ** -125


def test_oracle_token_by_token_is_the_same_as_at_once():
    rng = np.random.default_rng(0)
    K, V = rng.normal(size=(2, 1, 1, 100, 64))
    at_once, by_token = (so.Cache(1, 64, 64, [[1, 0]], 2) for _ in range(2))
    at_once.write(K, V, [0])
    for t in range(100):
        by_token.write(K[:, :, t:t + 1], V[:, :, t:t + 1], [t])
    for key, p in at_once.held.items():
        q = by_token.held[key]
        np.testing.assert_array_equal(p.k, q.k)
        np.testing.assert_array_equal(p.v, q.v)
        assert p.em == q.em and (p.mean == q.mean).all()
    out = at_once.attend(K[:, :, -1:], [100], None, 0.0, True)
    k, v, there = at_once.rows(0, 0, 0, 100)
    s = k @ K[0, 0, -1] / 8
    p = np.exp(s - s.max())
    assert there.all()
    np.testing.assert_allclose(out["O"][0, 0, 0], p @ v / p.sum(), rtol=1e-12)
    np.testing.assert_allclose(out["A"][0, 0, 0], p @ np.abs(v) / p.sum(), rtol=1e-12)


def test_zeros_are_outside_the_bound_of_the_attention():
    rng = np.random.default_rng(0)
    c = so.Cache(1, 64, 64, [range(4)], 4)
    K, V = rng.normal(size=(2, 1, 1, 256, 64))
    c.write(K, V, [0])
    r = c.attend(rng.normal(size=(1, 1, 3, 64)), [256], None, 0.0, False)
    assert ((np.abs(r["O"]) > 2.0 ** -8 * np.abs(r["O"]) + 2.0 ** -8 * r["A"]).mean(-1) > 0.9).all()


def test_pages_of_a_small_batch():
    # two sequences on blocks of four: the first grows over a border, the second is cut and gives a page back
    table, free, new, start, count, pos, slot = so.assign([[5, -1], [2, 7]], [9, 3], 2, [3, 6], [2, -3], 3, 4, 10)
    assert table.tolist() == [[5, 7], [2, -1]] and free == [9, 3] and new == [5, 3] and start == [3, 3] and count == [2, 0]
    assert pos.tolist() == [[3, 4, -1], [-1] * 3] and slot.tolist() == [[23, 28, -1], [-1] * 3]


def test_turning_by_a_quarter():
    x = np.zeros((1, 1, 1, 8))
    x[..., 0], x[..., 1], x[..., 4], x[..., 7] = 1, 2, 3, 5
    quarter = np.array([math.pi / 2] * 2)
    y, _ = so.rotate(x, np.ones((1, 1, 1), dtype=int), quarter, "interleaved", [2])
    np.testing.assert_allclose(y[0, 0, 0], [-2, 1, 0, 0, 3, 0, 0, 5], atol=1e-15)
    y, _ = so.rotate(x, np.ones((1, 1, 1), dtype=int), quarter, "half", [2], inverse=True)
    np.testing.assert_allclose(y[0, 0, 0], [0, 0, -1, -2, 3, 0, 0, 5], atol=1e-15)


# ---- sizes and frequencies -----------------------------------------------------------------------
ONE = 256                         # an address that is never read: validation fails first


def _cache(**kw):
    base = dict(batch=2, heads_kv=2, head_dim=128, block=64, max_blocks=10, pages=20, k_codes=ONE, v_codes=ONE, scales=ONE, k_mean=ONE, table=ONE)
    base.update(kw)
    return rb.rsa_cache(**base)


def _rows(heads=2, t=5, sb=5 * 2 * 128, sh=5 * 128, st=128):
    return rb.rsa_rows(heads, t, sb, sh, st)


def test_sizes(lib):
    c = _cache(k_codes=None, v_codes=None, scales=None, k_mean=None, table=None)
    assert rb.rsa_fourbit_bytes(c) == (20 * 2 * 64 * 68, 20 * 2 * 64 * 66, 20 * 2 * 16, 20 * 2 * 128)
    assert rb.rsa_fourbit_bytes(_cache(head_dim=64, block=128)) == (20 * 2 * 128 * 34, 20 * 2 * 128 * 34, 20 * 2 * 16, 20 * 2 * 64)
    assert lib.rsa_fourbit_bytes(None, None, None, None, None) == -1
    a = ctypes.c_size_t()
    assert lib.rsa_fourbit_workspace_bytes(ctypes.byref(_cache(max_blocks=5000)), ctypes.byref(_rows(heads=4)), 1, a) == 0 and a.value > 0
    assert lib.rsa_fourbit_workspace_bytes(ctypes.byref(c), ctypes.byref(_rows(heads=4)), -1, a) == -5
    assert lib.rsa_fourbit_workspace_bytes(ctypes.byref(c), ctypes.byref(_rows(heads=3)), 0, a) == -2


def test_frequencies(lib):
    n = 32
    plain = np.array([10000.0 ** (-j / n) for j in range(n)])
    f, factor = rb.rsa_rotary_frequencies(n)
    np.testing.assert_allclose(f, plain, rtol=1e-14)
    assert factor == 1
    np.testing.assert_allclose(rb.rsa_rotary_frequencies(n, 10000.0, rb.RSA_ROTARY_LINEAR, 4.0)[0], plain / 4, rtol=1e-14)
    f, factor = rb.rsa_rotary_frequencies(n, 10000.0, rb.RSA_ROTARY_BASE, 8.0)
    np.testing.assert_allclose([f[0], f[-1]], [1.0, plain[-1] / 8], rtol=1e-12)            # the slowest is stretched, the fastest is not
    f, factor = rb.rsa_rotary_frequencies(n, 10000.0, rb.RSA_ROTARY_PARTS, 8.0, 4096.0, 1.0, 32.0)
    turns = 4096 * plain / (2 * math.pi)
    f = np.array(f)
    np.testing.assert_allclose(f[turns >= 32], plain[turns >= 32], rtol=1e-14)
    np.testing.assert_allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    assert (np.diff(f) < 0).all() and abs(factor - (0.1 * math.log(8) + 1)) < 1e-7
    assert rb.rsa_rotary_frequencies(1, 10000.0, rb.RSA_ROTARY_BASE, 8.0)[0] == [1.0]
    for bad in ((0,), (513,), (4, 1.0), (4, math.inf), (4, 1e4, 4), (4, 1e4, -1), (4, 1e4, 1, 0.5), (4, 1e4, 1, math.nan), (4, 1e4, 3, 2.0, 0.0), (4, 1e4, 3, 2.0, 9.0, 2.0, 2.0),
                (2, 1e300, 2, 1e300)):
        with pytest.raises(rb.RsaError):
            rb.rsa_rotary_frequencies(*bad)


# ---- refusals ------------------------------------------------------------------------------------
BAD_CACHES = [(dict(batch=0), -2), (dict(heads_kv=0), -2), (dict(max_blocks=0), -2), (dict(pages=0), -2), (dict(head_dim=96), -3),
              (dict(block=32), -3), (dict(batch=40000), -3), (dict(pages=1 << 31), -3), (dict(max_blocks=1 << 26), -3)]


@pytest.mark.parametrize("kw,code", BAD_CACHES + [(dict(k_codes=None), -1), (dict(v_codes=None), -1), (dict(scales=None), -1), (dict(k_mean=None), -1),
                                                  (dict(table=None), -1), (dict(k_codes=264), -2), (dict(scales=260), -2), (dict(table=258), -2)])
def test_bad_caches_are_refused(lib, kw, code):
    c, r, R, by = _cache(**kw), _rows(), _rows(heads=4, sb=5 * 4 * 128), ctypes.byref
    assert lib.rsa_fourbit_write(by(c), by(r), ONE, ONE, ONE, None, None) == code
    assert lib.rsa_fourbit_read(by(c), by(r), ONE, None, ONE, 512, None) == code
    assert lib.rsa_fourbit_attn(by(c), by(R), ONE, ONE, None, 0.0, 0, None, None, 0, 0, ONE, None, None, 0, None) == code


@pytest.mark.parametrize("rows,code", [(None, -1), (dict(heads=0), -2), (dict(t=0), -2), (dict(st=64), -2), (dict(st=132), -2), (dict(sb=0), -2),
                                       (dict(sh=4), -2), (dict(heads=3), -2), (dict(t=1 << 28), -3)])
def test_bad_rows_are_refused(lib, rows, code):
    c, by = _cache(), ctypes.byref
    r = None if rows is None else by(_rows(**rows))
    assert lib.rsa_fourbit_attn(by(c), r, ONE, ONE, None, 0.0, 0, None, None, 0, 0, ONE, None, None, 0, None) == code
    assert lib.rsa_fourbit_write(by(c), r, ONE, ONE, ONE, None, None) == code
    assert lib.rsa_fourbit_read(by(c), r, ONE, None, ONE, 512, None) == code


def test_bad_arguments_are_refused(lib):
    c, r, R, by = _cache(), _rows(), _rows(heads=4), ctypes.byref
    write = lambda K=ONE, V=ONE, start=ONE, rows=r: lib.rsa_fourbit_write(by(c), by(rows), K, V, start, None, None)
    assert write(K=None) == -1 and write(V=None) == -1 and write(start=None) == -1 and write(K=264) == -2 and write(rows=R) == -2
    read = lambda K=ONE, V=512, start=ONE: lib.rsa_fourbit_read(by(c), by(r), start, None, K, V, None)
    assert read(K=None) == -1 and read(V=264) == -2 and read(V=ONE) == -5 and read(start=None) == -1

    def attn(Q=ONE, kv=ONE, scale=0.0, flags=0, idx=None, kept=None, group=0, n=0, O=ONE, ws=None, nws=0, cache=c, rows=R):
        return lib.rsa_fourbit_attn(by(cache), by(rows), Q, kv, None, scale, flags, idx, kept, group, n, O, None, ws, nws, None)
    assert attn(Q=None) == -1 and attn(kv=None) == -1 and attn(O=None) == -1 and attn(idx=ONE) == -1 and attn(kept=ONE) == -1
    assert attn(Q=264) == -2 and attn(O=264) == -2 and attn(flags=2) == -5
    for scale in (-1.0, math.nan, math.inf, 3e38, -1e-45):
        assert attn(scale=scale) == -5
    assert attn(idx=ONE, kept=ONE, group=0, n=4) == -5 and attn(idx=ONE, kept=ONE, group=1, n=0) == -5
    assert attn(ws=ONE, nws=16, cache=_cache(max_blocks=100)) == -4 and attn(ws=264, nws=1 << 30) == -4
    # more workgroups than a launch takes: refused by the host
    many = _rows(heads=4, t=1 << 23, sb=(1 << 23) * 4 * 128, sh=(1 << 23) * 128)
    assert attn(idx=ONE, kept=ONE, group=1, n=4, rows=many) == -3


def test_bad_pages_are_refused(lib):
    def call(t=1, kv=0x1000, add=0x2000, shared=None, fc=0x3000, new=0x4000, left=0x5000, start=0x6000, count=0x7000, pos=None, slots=None, **kw):
        base = dict(batch=2, max_blocks=4, block=64, pages=8, table=0x8000, free_pages=0x9000)
        base.update(kw)
        return lib.rsa_cache_assign(ctypes.byref(rb.rsa_pages(**base)), t, kv, add, shared, fc, new, left, start, count, pos, slots, None)
    assert lib.rsa_cache_assign(None, 1, *[ONE] * 10, None) == -1
    for kw in (dict(batch=0), dict(max_blocks=0), dict(block=0), dict(pages=0), dict(t=0)):
        assert call(**kw) == -2, kw
    for kw in (dict(batch=65536), dict(pages=1 << 31), dict(max_blocks=1 << 26, block=64), dict(t=1 << 27), dict(batch=65535, t=1 << 13), dict(batch=65535, max_blocks=1 << 16, block=1)):
        assert call(**kw) == -3, kw
    for kw in (dict(table=None), dict(free_pages=None), dict(kv=None), dict(add=None), dict(fc=None), dict(new=None), dict(left=None), dict(start=None), dict(count=None)):
        assert call(**kw) == -1, kw
    for kw in (dict(table=0x8002), dict(kv=0x1001), dict(pos=2), dict(slots=0x1004), dict(shared=2)):
        assert call(**kw) == -2, kw
    for kw in (dict(start=0x7000), dict(new=0x2000), dict(start=0x1000), dict(count=0x3000), dict(left=0x4000), dict(free_pages=0x8000), dict(start=0x2000),
               dict(shared=0x4000), dict(new=0x3000), dict(left=0x1000), dict(table=0x1000)):
        assert call(**kw) == -5, kw
    # the maps of the new rows over anything that is read or written
    for at in (0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000, 0xa000):
        assert call(shared=0xa000, pos=at) == -5 and call(shared=0xa000, slots=at) == -5, at
    assert call(pos=0xb000, slots=0xb000) == -5


def test_bad_rotary_is_refused(lib):
    by = ctypes.byref

    def call(rows=_rows(), Q=0x1000, Qr=0x2000, rows_k=None, K=None, Kr=None, pos=None, start=None, count=None, flags=0, batch=2, **kw):
        base = dict(head_dim=128, pairs=64, interleaved=0, axes=1, axis_pairs=(ctypes.c_int32 * 3)(*kw.pop("axis_pairs", (64, 0, 0))), factor=1.0, freq=0x3000)
        base.update(kw)
        return lib.rsa_rotary_apply(by(rb.rsa_rotary(**base)), batch, None if rows is None else by(rows), Q, Qr, None if rows_k is None else by(rows_k), K, Kr,
                                    pos, start, count, flags, None)
    assert lib.rsa_rotary_apply(None, 1, by(_rows()), ONE, ONE, None, None, None, None, None, None, 0, None) == -1
    for kw in (dict(rows=None), dict(Q=None), dict(Qr=None), dict(freq=None), dict(rows_k=_rows()), dict(rows_k=_rows(), K=0x4000), dict(axes=2, axis_pairs=(60, 4, 0))):
        assert call(**kw) == -1, kw
    for kw in (dict(head_dim=0), dict(head_dim=124), dict(pairs=0, axis_pairs=(0, 0, 0)), dict(pairs=65, axis_pairs=(65, 0, 0)), dict(axes=0), dict(axes=4),
               dict(axis_pairs=(63, 0, 0)), dict(axes=3, axis_pairs=(66, -1, -1), pos=ONE), dict(axes=2, axis_pairs=(1 << 31 - 1, 64, 0), pos=ONE), dict(batch=0),
               dict(rows=_rows(t=0)), dict(rows=_rows(heads=0)), dict(rows=_rows(st=64)), dict(rows=_rows(st=132)), dict(rows=_rows(sb=4)), dict(rows=_rows(sh=0)),
               dict(Q=0x1008), dict(Qr=0x2002), dict(freq=0x3004), dict(pos=2), dict(start=2), dict(count=1),
               dict(rows_k=_rows(t=4), K=0x4000, Kr=0x5000), dict(rows_k=_rows(), K=0x4008, Kr=0x5000)):
        assert call(**kw) == -2, kw
    for kw in (dict(head_dim=1032, rows=_rows(st=2048)), dict(rows=_rows(t=1 << 28)), dict(rows=_rows(t=1 << 26), batch=3)):
        assert call(**kw) == -3, kw
    for kw in (dict(factor=-1.0), dict(factor=math.nan), dict(factor=math.inf), dict(flags=2), dict(rows_k=_rows(), K=0x4000, Kr=0x2000),
               dict(rows_k=_rows(), K=0x4000, Kr=0x1000), dict(rows_k=_rows(), K=0x2000, Kr=0x5000)):
        assert call(**kw) == -5, kw


def test_binding_refuses_cpu_tensors_and_wrong_buffers(lib):
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    args = dict(k_codes=u8(4, 2, 64 * 34), v_codes=u8(4, 2, 64 * 34), scales=torch.zeros(4, 2, 4), k_mean=torch.zeros(4, 2, 64, dtype=torch.int8),
                table=torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="device tensors only"):
        rb.fourbit_of(**args, block=64)
    for name, bad in (("k_codes", u8(4, 2, 64 * 64)), ("v_codes", u8(4, 2, 64 * 32)), ("scales", torch.zeros(4, 2, 2)), ("k_mean", torch.zeros(4, 2, 64)),
                      ("table", torch.zeros(1, 4))):
        with pytest.raises(ValueError):
            rb.fourbit_of(**{**args, name: bad}, block=64)
    with pytest.raises(ValueError):
        rb.pages_of(torch.zeros(2, 4), torch.zeros(4, dtype=torch.int32), 64)
    with pytest.raises(RuntimeError, match="device tensors only"):
        rb.pages_of(torch.zeros(2, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 64)
    f = torch.ones(8, dtype=torch.float64)
    for bad in (dict(freq=f.float()), dict(freq=f[::2]), dict(freq=f, pairing="pairs"), dict(freq=f, axis_pairs=[4, 3]), dict(freq=f, axis_pairs=[2] * 4),
                dict(freq=f, axis_pairs=[9, -1])):
        with pytest.raises(ValueError):
            rb.make_rotary(**bad)
    with pytest.raises(RuntimeError, match="device tensors only"):
        rb.make_rotary(f)


def test_rotary_records_that_a_call_would_refuse_are_refused_when_they_are_made(lib):
    """A step moves its lengths on before it turns anything, so a record that rsa_rotary_apply refuses must not get that far."""
    f = torch.ones(8, dtype=torch.float64)
    for bad in (dict(factor=-1.0), dict(factor=math.nan), dict(factor=math.inf), dict(factor=1e39), dict(freq=torch.ones(0, dtype=torch.float64))):
        with pytest.raises(ValueError):
            rb.make_rotary(**{**dict(freq=f), **bad})
    record = lambda **kw: rb.rsa_rotary(**{**dict(head_dim=0, pairs=8, interleaved=0, axes=1, axis_pairs=(ctypes.c_int32 * 3)(8, 0, 0), factor=1.0, freq=ONE), **kw})
    for bad in (dict(factor=-1.0), dict(factor=math.nan), dict(factor=1e39), dict(pairs=0)):
        with pytest.raises(ValueError):
            rb.Rotary(record(**bad), f)
    for fine in (0.0, 1.2):
        assert rb.Rotary(record(factor=fine), f).desc.factor == np.float32(fine)


def test_a_shared_prefix_over_other_arguments_is_refused(lib):
    """It is written where pages are taken below it."""
    pages = rb.rsa_pages(batch=2, max_blocks=4, block=64, pages=8, table=0x8000, free_pages=0x9000)
    for at in range(0x1000, 0xc000, 0x1000):
        args = [0x1000, 0x2000, at, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0xa000, 0xb000]
        assert lib.rsa_cache_assign(ctypes.byref(pages), 1, *args, None) == -5, hex(at)
    in_place = [0x1000, 0x2000, 0x1000, 0x3000, 0x1000, 0x3000, 0x6000, 0x7000, None, None]
    assert lib.rsa_cache_assign(ctypes.byref(pages), 1, *in_place, None) == -5


def test_pages_below_a_shared_prefix_are_the_sequences_own():
    """Two sequences on a prefix of two pages; the second goes back to the first page, on, and back again: what it took comes back."""
    table, free, kv, shared = [[0, 1, -1], [0, 1, 2]], [3, 4], [128, 192], [2, 2]
    for add, want_free, want_shared, row in ((-128, [3, 4, 2], 2, [0, -1, -1]), (128, [3], 1, [0, 2, 4]), (-128, [3, 2, 4], 1, [0, -1, -1])):
        table, free, kv, *_ = so.assign(table, free, len(free), kv, [0, add], 128, 64, 5, shared)
        assert free == want_free and shared == [2, want_shared] and table.tolist()[1] == row


def test_no_token_goes_into_a_shared_page():
    """A sequence that ends inside a block of its prefix is not served; at the block's border, or with that block its own, it is."""
    for kv, shared, served in ((70, 2, False), (64, 2, True), (128, 2, True), (130, 2, True), (70, 1, True), (1, 1, False), (0, 2, True), (70, -1, True)):
        n = -(-kv // 64)
        row = list(range(n)) + [-1] * (4 - n)
        table, free, new, start, count, pos, slot = so.assign([row], [7, 8], 2, [kv], [1], 1, 64, 9, [shared])
        assert (count, new) == (([1], [kv + 1]) if served else ([0], [kv])) and (served or (table.tolist() == [row] and free == [7, 8] and pos == [[-1]] and slot == [[-1]]))
