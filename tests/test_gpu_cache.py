"""The 8-bit key/value cache on the GPU against its oracle (oracle/cache_oracle.py).

What a write leaves, what is read back, the means behind the scores and the lists are exact: compared bit for bit. Outputs of
the attention are held to a bound made of its roundings, for each element:

  |O - O64| <= 2^-8 |O64|                         the output in bf16: half a step
             + (2^-11 + 2 e_s + 4 n 2^-24) A      P in fp16: half a step of 2^-11 of each p, of 2^-25 below 2^-14; scores off by e_s change
                                                  p by e_s of itself, above and below the division; sums of n terms in 32 bits, each way
  e_s = (d + 16) 2^-24 max_j sum|q||k_j| * scale  the dot product in 32 bits and the few operations behind it
  |lse - lse64| <= 2 e_s + 4 n 2^-24 + 2^-21 max(1, |lse|)

with A = sum min(max(p, 2^-14), 2^11 p) |v| over the same keys and over sum p, the largest p being 1 (oracle: vmax is 0).
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_19835_amd import binding as rb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf16(x, layout="bhtd"):
    x = torch.as_tensor(np.ascontiguousarray(x)).to(torch.float32).to(torch.bfloat16).to(DEV)
    return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if layout == "bthd" else x.contiguous()


def f64(x):
    return x.detach().cpu().double().numpy()


def i32(x):
    return None if x is None else torch.tensor(list(x), dtype=torch.int32, device=DEV)


def video_like(rng, *shape, spread=0.0):
    """Rows with a slow drift along the tokens, and tokens whose size differs by e^spread."""
    b, h, t, d = shape
    x = rng.normal(size=shape) * 0.6 + np.cumsum(rng.normal(size=shape), axis=2) * 0.15
    return x * np.exp(rng.normal(size=(b, h, t, 1)) * spread)


class Pair:
    """A cache on the GPU and the oracle's, with the same table; uninitialised pages hold the code of NaN everywhere."""

    def __init__(self, batch, hk, d, block, max_blocks, seed=0, table=None, pages=None):
        n = batch * max_blocks
        self.rng = np.random.default_rng(seed)
        if table is None:
            pages = pages or n + 2
            table = self.rng.permutation(pages)[:n].reshape(batch, max_blocks)
        self.gpu = rb.allocate_cache(batch, hk, d, block, pages, max_blocks, DEV)
        self.gpu.k_codes.fill_(0x7f)
        self.gpu.v_codes.fill_(0xff)
        self.gpu.scales.fill_(float("nan"))
        self.gpu.k_mean.fill_(77)
        self.gpu.table.copy_(torch.as_tensor(np.asarray(table, dtype=np.int32)))
        self.ref = co.Cache(hk, d, block, table, pages)
        self.batch, self.hk, self.d, self.block = batch, hk, d, block

    def write(self, K, V, start, count=None, layout="bhtd", stream=None):
        K, V = bf16(K, layout), bf16(V, layout)
        rb.rsa_cache_write(self.gpu, rb.make_rows(K), K, V, i32(start), i32(count), stream)
        self.ref.write(f64(K), f64(V), start, count)

    def fill(self, lens, spread=0.0):
        t = max(max(lens), 1)
        K = video_like(self.rng, self.batch, self.hk, t, self.d, spread=spread)
        V = self.rng.normal(size=K.shape)
        self.write(K, V, [0] * self.batch, lens)

    def check_pages(self):
        """Every page that was written, bit for bit; no other page touched."""
        scales, mean = self.gpu.scales.cpu().numpy(), self.gpu.k_mean.cpu().numpy()
        t, ch = np.arange(self.block)[:, None], np.arange(self.d)[None]
        at_k = ((t // 16 * (self.d // 64) + ch // 64) * 4 + ch % 64 // 16) * 256 + t % 16 * 16 + ch % 16
        at_v = ((t // 64 * (self.d // 16) + ch // 16) * 4 + t % 16 // 4) * 256 + ch % 16 * 16 + t % 64 // 16 * 4 + t % 4
        k, v = (x.cpu().view(torch.float8_e4m3fn).double().numpy()[:, :, at] for x, at in ((self.gpu.k_codes, at_k), (self.gpu.v_codes, at_v)))
        for page in range(scales.shape[0]):
            for h in range(self.hk):
                p = self.ref.held.get((page, h))
                if p is None:
                    assert np.isnan(scales[page, h]).all() and (mean[page, h] == 77).all() and np.isnan(k[page, h]).all()
                    continue
                assert scales[page, h].tolist() == [2.0 ** p.ek, 2.0 ** p.ev, 2.0 ** p.em, 0.0]
                np.testing.assert_array_equal(k[page, h] * 2.0 ** p.ek, p.k)
                np.testing.assert_array_equal(v[page, h] * 2.0 ** p.ev, p.v)
                np.testing.assert_array_equal(mean[page, h], p.mean)


def attend(pair, Q, kv_len, q_len=None, scale=0.0, causal=False, lists=None, group=0, layout="bhtd", ws=True, stream=None, list_len=0):
    """rsa_cache_attn on Q (numpy) -> (outputs, lse) as numpy, rows that are no query checked to be untouched."""
    Qd = bf16(Q, layout)
    O = torch.full_like(Qd, 7.0)
    lse = torch.full(Qd.shape[:3], 7.0, dtype=torch.float32, device=DEV)
    rows = rb.make_rows(Qd)
    idx = kept = None
    if lists is not None:
        groups = -(-Q.shape[2] // group)
        n = max(1, list_len, max(len(x) for x in lists.values()))
        idx = torch.full((pair.batch, pair.hk, groups, n), -1, dtype=torch.int32)
        kept = torch.zeros(pair.batch, pair.hk, groups, dtype=torch.int32)
        for (b, h, g), x in lists.items():
            idx[b, h, g, :len(x)] = torch.tensor(x, dtype=torch.int32)
            kept[b, h, g] = len(x)
        idx, kept = idx.to(DEV), kept.to(DEV)
    scratch = None
    if ws:
        _, n = rb.rsa_cache_workspace_bytes(pair.gpu, rows, group)
        scratch = torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device=DEV)     # NaN wherever it is read before it is written
    rb.rsa_cache_attn(pair.gpu, rows, Qd, i32(kv_len), i32(q_len), scale, rb.RSA_CACHE_CAUSAL if causal else 0, idx, kept, group, O, lse, scratch, stream)
    torch.cuda.synchronize()
    ref = pair.ref.attend(f64(Qd), kv_len, q_len, scale, causal, lists, group)
    return f64(O), lse.cpu().double().numpy(), ref


def compare(O, lse, ref, d):
    isq = ref["isq"]
    assert (O[~isq] == 7.0).all() and (lse[~isq] == 7.0).all(), "rows behind the last query were written"
    O, lse = O[isq], lse[isq]
    want, A, want_lse, S, n, vmax = (ref[k][isq] for k in ("O", "A", "lse", "S", "n", "vmax"))
    empty = n == 0
    assert (O[empty] == 0).all() and np.isneginf(lse[empty]).all()
    O, lse, want, A, want_lse, S, n, vmax = (x[~empty] for x in (O, lse, want, A, want_lse, S, n, vmax))
    assert np.array_equal(np.isnan(O), np.isnan(want)) and np.array_equal(np.isnan(lse), np.isnan(want_lse))
    es = (d + 16) * 2.0 ** -24 * S
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * es + 4 * n * 2.0 ** -24)[:, None] * A + (n * 2.0 ** -24 * vmax)[:, None]
    ok = ~np.isnan(want)
    worst = (np.abs(O - want)[ok] / np.maximum(bound[ok], 1e-30)).max(initial=0)
    fine = ~np.isnan(want_lse)
    lb = 2 * es + 4 * n * 2.0 ** -24 + 2.0 ** -21 * np.maximum(1, np.abs(np.where(fine, want_lse, 0)))
    worst_lse = (np.abs(lse - want_lse)[fine] / lb[fine]).max(initial=0)
    print(f"of the bound: outputs {worst:.2f}, lse {worst_lse:.2f}")
    assert worst <= 1 and worst_lse <= 1


# ---- writing and reading -------------------------------------------------------------------------
@pytest.mark.parametrize("d,block,layout", [(64, 64, "bhtd"), (64, 128, "bthd"), (128, 64, "bthd"), (128, 128, "bhtd")])
def test_write_in_pieces(d, block, layout):
    """Ragged pieces: inside a block, across several, one token, none, more than there are rows, before the start."""
    p = Pair(3, 2, d, block, 6)
    pos = np.zeros(3, dtype=int)
    for step, (t, count) in enumerate([(5, [5, 1, 0]), (1, [1, 1, 1]), (200, [200, 3, 131]), (block, None), (70, [64, -3, 99]), (2, [2, 2, 2])]):
        K = video_like(p.rng, 3, 2, t, d) * 2.0 ** (step - 2)                  # later tokens are larger: scales rise
        p.write(K, p.rng.normal(size=K.shape) * 2.0 ** (3 - step), pos.tolist(), count, layout)
        pos += np.clip(count if count is not None else [t] * 3, 0, t)
        p.check_pages()
    p.write(video_like(p.rng, 3, 2, 9, d), video_like(p.rng, 3, 2, 9, d), [-1, 30, block + 2], None, layout)   # back to an earlier length
    p.check_pages()


@pytest.mark.parametrize("d,block", [(64, 64), (128, 128), (128, 64)])
def test_token_by_token(d, block):
    p = Pair(2, 1, d, block, 2)
    K = video_like(p.rng, 2, 1, block + 5, d, spread=2.0)
    V = p.rng.normal(size=K.shape) * np.exp(p.rng.normal(size=(2, 1, block + 5, 1)) * 2)
    for t in range(block + 5):
        p.write(K[:, :, t:t + 1], V[:, :, t:t + 1], [t, t])
    p.check_pages()


def test_write_at_the_ends_of_the_range():
    """Zeros, the smallest and largest bf16, infinities, NaN, and every code boundary."""
    p = Pair(1, 1, 64, 64, 8)
    edge = np.zeros((1, 1, 8 * 64, 64))
    edge[0, 0, 64:128] = np.ldexp(p.rng.normal(size=(64, 64)), -130)
    edge[0, 0, 128:192] = np.ldexp(1.0 + p.rng.integers(0, 128, size=(64, 64)) / 128, 127)
    edge[0, 0, 192:256] = p.rng.normal(size=(64, 64))
    edge[0, 0, 200, 3], edge[0, 0, 201, 4], edge[0, 0, 202, 5] = np.inf, -np.inf, np.nan
    edge[0, 0, 256:320] = np.nan
    edge[0, 0, 320:384] = np.linspace(-448, 448, 4096).reshape(64, 64)
    edge[0, 0, 384:448] = np.ldexp(np.linspace(-64, 64, 4096), -9).reshape(64, 64)
    edge[0, 0, 384, 0] = 448
    edge[0, 0, 448:] = np.where(p.rng.random((64, 64)) < 0.5, 225, -225)
    x = torch.as_tensor(edge).float().clamp(-3.3895313892515355e38, 3.3895313892515355e38)
    x = torch.where(torch.isinf(torch.as_tensor(edge).float()) & (torch.as_tensor(np.arange(512)).view(1, 1, -1, 1) > 192), torch.as_tensor(edge).float(), x)
    p.write(x.numpy(), x.flip(2).numpy(), [0])
    p.check_pages()


def test_write_passes_over_what_is_no_page():
    table = [[2, -1, 9, 0], [7, 1, 3, -5]]                      # pages 0..3 exist
    p = Pair(2, 2, 64, 64, 4, table=table, pages=4)
    K = video_like(p.rng, 2, 2, 300, 64)                        # more than the table holds, too
    p.write(K, K[:, :, ::-1], [0, 30])
    p.check_pages()
    R, S = bf16(np.full((2, 2, 300, 64), 7.0)), bf16(np.full((2, 2, 300, 64), 7.0))
    rb.rsa_cache_read(p.gpu, rb.make_rows(R), i32([0, 30]), None, R, S)
    for b, s in enumerate((0, 30)):
        for h in range(2):
            k, v, there = p.ref.rows(b, h, s, s + 300)
            np.testing.assert_array_equal(f64(R)[b, h], np.where(there[:, None], k, 7.0))
            np.testing.assert_array_equal(f64(S)[b, h], np.where(there[:, None], v, 7.0))


@pytest.mark.parametrize("d,block,layout", [(64, 128, "bhtd"), (128, 64, "bthd"), (128, 128, "bthd"), (64, 64, "bhtd")])
def test_read_back(d, block, layout):
    p = Pair(3, 2, d, block, 4)
    p.fill([4 * block, 2 * block + 3, 1])
    t = 2 * block + 9
    start, count = [block - 3, 2, 0], [t, 2 * block + 1, 1]
    K, V = bf16(np.full((3, 2, t, d), 7.0), layout), bf16(np.full((3, 2, t, d), 7.0), layout)
    rb.rsa_cache_read(p.gpu, rb.make_rows(K), i32(start), i32(count), K, V)
    for b in range(3):
        for h in range(2):
            k, v, _ = p.ref.rows(b, h, start[b], start[b] + count[b])
            for got, want in ((K, k), (V, v)):
                np.testing.assert_array_equal(f64(got)[b, h, :count[b]], want)
                assert (f64(got)[b, h, count[b]:] == 7.0).all()


# ---- selection -----------------------------------------------------------------------------------
def select(p, Q, kv_len, q_len, group, keep, first, last, causal, layout="bhtd", ws=True):
    Qd = bf16(Q, layout)
    groups, mb = -(-Q.shape[2] // group), p.gpu.desc.max_blocks
    n = min(mb, max(keep, first + last + -(-group // p.block) + 1))
    idx = torch.full((p.batch, p.hk, groups, n), 12345, dtype=torch.int32, device=DEV)
    kept = torch.full((p.batch, p.hk, groups), 12345, dtype=torch.int32, device=DEV)
    rows = rb.make_rows(Qd)
    scratch = torch.full((max(256, rb.rsa_cache_workspace_bytes(p.gpu, rows, group)[0]),), 0xff, dtype=torch.uint8, device=DEV) if ws else None
    rb.rsa_cache_select(p.gpu, rows, Qd, i32(kv_len), i32(q_len), group, keep, first, last, rb.RSA_CACHE_CAUSAL if causal else 0, idx, kept, scratch)
    want = p.ref.select(f64(Qd), kv_len, q_len, group, keep, first, last, causal)
    idx, kept = idx.cpu().numpy(), kept.cpu().numpy()
    for (b, h, g), x in want.items():
        assert kept[b, h, g] == len(x), (b, h, g)
        assert idx[b, h, g].tolist() == x + [-1] * (n - len(x)), (b, h, g)
    return want


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,block,G,t,group,keep,first,last,causal,layout", [
    (64, 64, 1, 1, 1, 3, 0, 1, True, "bhtd"), (128, 128, 4, 1, 1, 5, 1, 2, True, "bhtd"), (128, 64, 5, 7, 1, 4, 1, 0, True, "bthd"),
    (128, 64, 1, 150, 64, 6, 0, 1, True, "bthd"), (64, 128, 2, 131, 50, 2, 2, 3, False, "bhtd"), (128, 128, 3, 40, 128, 100, 0, 0, False, "bhtd"),
    (64, 64, 2, 5, 1 << 30, 3, 0, 1, True, "bhtd"), (64, 64, 1, 9, 4, 1, 0, 0, True, "bhtd")])
def test_select(d, block, G, t, group, keep, first, last, causal, layout, ws):
    p = Pair(3, 2, d, block, 20)
    lens = [20 * block, 11 * block + 7, t]
    p.fill(lens)
    Q = video_like(p.rng, 3, 2 * G, t, d)
    select(p, Q, lens, None, group, keep, first, last, causal, layout, ws)
    select(p, Q, lens, [t, max(t - 2, 0), 0], group, keep, first, last, causal, layout, ws)


@pytest.mark.parametrize("ws", [True, False])
def test_select_ties_and_odd_queries(ws):
    """Blocks of the same keys score the same: the lower ones go first. Queries with NaN and infinities, and all zero ones."""
    p = Pair(2, 1, 64, 64, 30)
    K = np.repeat(p.rng.normal(size=(2, 1, 3, 64)), 640, axis=2)               # thirty blocks of three kinds
    p.write(K, K, [0, 0], [1920, 1000])
    Q = p.rng.normal(size=(2, 2, 3, 64))
    Q[0, 0, 1] = 0
    Q[0, 1, 1] = 0
    Q[1, 0, 0, 5], Q[1, 1, 2, 6], Q[1, 1, 2, 7] = np.nan, np.inf, -np.inf
    for keep in (1, 7, 12, 29, 30):
        select(p, Q, [1920, 1000], None, 1, keep, 0, 1, True, ws=ws)


@pytest.mark.parametrize("ws", [True, False])
def test_select_where_pages_are_missing(ws):
    table = np.arange(20).reshape(2, 10)
    table[0, 3], table[0, 9], table[1, 0], table[1, 5] = -1, 1000, 77, -3
    p = Pair(2, 2, 128, 64, 10, table=table, pages=20)
    p.fill([640, 500])
    select(p, p.rng.normal(size=(2, 4, 2, 128)), [640, 500], None, 1, 6, 1, 2, True, ws=ws)
    select(p, p.rng.normal(size=(2, 4, 2, 128)), [0, 1], [2, 2], 1, 6, 1, 2, True, ws=ws)       # a sequence without tokens; positions before the first


@pytest.mark.parametrize("stray", [-1.0, 0.0, 1e-45, float("nan"), float("inf"), -3e38])
def test_select_whatever_a_page_holds(stray):
    """Scales of means as they may stand in memory that was never written: a block counts by its entry in the table, and as many as asked
    for are listed."""
    table = np.random.default_rng(2).permutation(90).reshape(1, 90)
    table[0, 11] = -1
    p = Pair(1, 2, 128, 64, 90, table=table, pages=90)
    p.fill([90 * 64])
    p.gpu.scales[torch.as_tensor(table[0, ::3].copy()).long().to(DEV), :, 2] = stray
    Q = bf16(p.rng.normal(size=(1, 2, 1, 128)))
    for keep in (30, 89, 90):
        buf = torch.full((2 * 90 + 100,), 12345, dtype=torch.int32, device=DEV)
        idx, kept = buf[:180].view(1, 2, 1, 90), torch.zeros(1, 2, 1, dtype=torch.int32, device=DEV)
        rb.rsa_cache_select(p.gpu, rb.make_rows(Q), Q, i32([90 * 64]), None, 1, keep, 0, 0, 0, idx, kept)
        assert kept.flatten().tolist() == [min(keep, 89)] * 2 and (buf[180:] == 12345).all()
        for row in idx.view(2, 90).tolist():
            own = row[:min(keep, 89)]
            assert own == sorted(set(own)) and 0 <= own[0] and own[-1] < 90 and 11 not in own and row[len(own):] == [-1] * (90 - len(own))


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("blocks,keep", [(1000, 100), (16384, 700)])
def test_select_long(blocks, keep, ws):
    """Many blocks, means and scales drawn directly (a page for each of the 300 kinds)."""
    p = Pair(1, 2, 128, 64, blocks, table=np.random.default_rng(1).integers(0, 300, size=(1, blocks)), pages=300)
    for page in range(300):
        for h in range(2):
            q = p.ref.held.setdefault((page, h), co.Page(64, 128))
            q.mean, q.em = p.rng.integers(-127, 128, size=128), int(p.rng.integers(-100, 20))
    p.gpu.k_mean.copy_(torch.as_tensor(np.array([[p.ref.held[i, h].mean for h in range(2)] for i in range(300)])))
    p.gpu.scales.copy_(torch.as_tensor(np.array([[[1, 1, 2.0 ** p.ref.held[i, h].em, 0] for h in range(2)] for i in range(300)])))
    select(p, p.rng.normal(size=(1, 2, 3, 128)), [blocks * 64], None, 1, keep, 1, 1, True, ws=ws)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,blocks,keep,most", [(128, 10, 3, 1), (64, 40, 7, 3), (128, 200, 9, 3), (64, 600, 50, 1), (128, 2000, 33, 3), (64, 4200, 90, 3)])
def test_select_among_the_smallest_scores(d, blocks, keep, most, ws):
    """Mean keys of 0 .. 3 times 2^-100 in a channel where the query's code is 1: scores 2^-122 apart, the least there are."""
    p = Pair(1, 2, d, 64, blocks, table=np.arange(blocks).reshape(1, blocks) % 7, pages=7)
    K = np.zeros((1, 2, 7 * 64, d))
    K[..., 1] = np.repeat(p.rng.permutation(7) % (most + 1), 64) * 2.0 ** -100
    p.write(K, K, [0])
    p.check_pages()
    Q = np.zeros((1, 4, 3, d))
    Q[..., 0], Q[..., 1] = 127, 1                                              # (four heads, two to a key/value head: sums of 254 and 2)
    guard = 500
    Qd, kv = bf16(Q), i32([blocks * 64])
    n = keep + 1
    buf = torch.full((2 * 3 * n + guard,), 12345, dtype=torch.int32, device=DEV)
    idx, kept = buf[:2 * 3 * n].view(1, 2, 3, n), torch.zeros(1, 2, 3, dtype=torch.int32, device=DEV)
    rows = rb.make_rows(Qd)
    scratch = torch.empty(max(256, rb.rsa_cache_workspace_bytes(p.gpu, rows, 1)[0]), dtype=torch.uint8, device=DEV) if ws else None
    rb.rsa_cache_select(p.gpu, rows, Qd, kv, None, 1, keep, 0, 0, 0, idx, kept, scratch)
    want = p.ref.select(f64(Qd), [blocks * 64], None, 1, keep, 0, 0, False)
    assert (buf[2 * 3 * n:] == 12345).all()
    for (b, h, g), x in want.items():
        assert int(kept[b, h, g]) == keep and idx[b, h, g].tolist() == x + [-1], (b, h, g)


# ---- attention -----------------------------------------------------------------------------------
SHAPES = [  # d, block, G, t, lens, q_len, causal
    (64, 64, 1, 1, [1], None, True),                              # one key
    (64, 64, 1, 1, [65, 1000, 64], None, False),
    (128, 64, 4, 1, [700, 1, 130], None, True),
    (128, 128, 8, 1, [129, 1300, 128], None, True),
    (64, 128, 5, 3, [200, 3, 500], [3, 3, 2], True),              # heads that fill no tile
    (128, 128, 1, 17, [300, 17, 900], [17, 5, 16], True),
    (128, 64, 2, 33, [33, 400, 64], None, True),                  # drafts and prompts
    (128, 128, 1, 130, [130, 600, 257], [130, 1, 99], True),
    (64, 64, 3, 70, [100, 640, 71], None, False),
    (128, 64, 16, 2, [250, 90, 3], None, True),
    (64, 128, 1, 200, [200, 1000, 333], [200, 150, 0], True),
    (128, 128, 2, 150, [1000, 150, 500], None, False),
    (128, 64, 4, 1, [3000, 1, 1700], None, True),                 # long enough that the key axis is split
    (64, 128, 1, 5, [2600, 5, 2049], [5, 4, 5], True),
    (128, 128, 3, 9, [2000, 77, 1930], None, False),
    (64, 64, 1, 100, [2100, 100, 1000], [100, 7, 64], True),
]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,block,G,t,lens,q_len,causal", SHAPES)
def test_attention(d, block, G, t, lens, q_len, causal, ws):
    b = len(lens)
    p = Pair(b, 2, d, block, -(-max(lens) // block) + 1)
    p.fill(lens, spread=0.5)
    Q = video_like(p.rng, b, 2 * G, t, d)
    compare(*attend(p, Q, lens, q_len, causal=causal, layout="bthd" if t % 2 else "bhtd", ws=ws), d)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,block,G,t,group,causal", [(64, 64, 1, 1, 1, True), (128, 64, 4, 1, 1, True), (128, 128, 3, 5, 1, True),
                                                      (128, 128, 1, 200, 128, False), (128, 64, 2, 90, 64, True), (64, 128, 1, 77, 20, True),
                                                      (128, 128, 1, 129, 1 << 30, False)])
def test_attention_over_lists(d, block, G, t, group, causal, ws):
    p = Pair(2, 2, d, block, 9)
    lens = [9 * block - 5, 4 * block + max(0, t - 4 * block)]
    p.fill(lens)
    Q = video_like(p.rng, 2, 2 * G, t, d)
    q_len = [t, max(1, t - 3)]
    lists = p.ref.select(f64(bf16(Q)), lens, q_len, group, 4, 1, 1, causal)
    compare(*attend(p, Q, lens, q_len, causal=causal, lists=lists, group=min(group, t), ws=ws), d)
    # any list is taken: no order, entries that are none, blocks behind the last visible one, empty ones, a block twice
    odd = {k: [[], [7, 0, 100, -1, 2], [3, 3], [8, 1, -2147483648, 2147483647]][i % 4] for i, k in enumerate(lists)}
    compare(*attend(p, Q, lens, q_len, causal=causal, lists=odd, group=min(group, t), ws=ws, list_len=70), d)   # longer than the table, too


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("t,group,G", [(1, 1, 4), (20, 20, 1), (90, 90, 1)])
def test_attention_over_long_lists(t, group, G, ws):
    """Forty of fifty blocks, in any order, some without a page."""
    table = np.random.default_rng(3).permutation(60)[:50].reshape(1, 50)
    table[0, 7], table[0, 33] = -1, 60
    p = Pair(1, 1, 128, 64, 50, table=table, pages=60)
    p.fill([3150])
    Q = video_like(p.rng, 1, G, t, 128)
    lists = {(0, 0, 0): p.rng.permutation(50)[:40].tolist()}
    compare(*attend(p, Q, [3150], causal=True, lists=lists, group=group, ws=ws), 128)


def test_attention_passes_over_what_is_no_page():
    table = np.arange(20).reshape(2, 10)
    table[0, 3], table[0, 9], table[1, 0], table[1, 5] = -1, 1000, 77, -3
    p = Pair(2, 2, 128, 64, 10, table=table, pages=20)
    p.fill([640, 500])
    Q = p.rng.normal(size=(2, 4, 3, 128))
    compare(*attend(p, Q, [640, 500], causal=True), 128)
    compare(*attend(p, Q, [64 * 3 + 1, 30], causal=False), 128)               # the only visible block of the second is missing
    compare(*attend(p, Q, [0, 2], [3, 3], causal=True), 128)                  # no token; positions before the first
    compare(*attend(p, Q, [5000, -7], [3, 3], causal=False), 128)             # longer than the table; negative


@pytest.mark.parametrize("t,G", [(4, 2), (40, 1), (140, 1)])
def test_nan_stays_with_the_rows_that_see_it(t, G):
    """NaN among values and among keys of single tokens: causal rows before them are unharmed."""
    p = Pair(2, 1, 128, 64, 4)
    K, V = p.rng.normal(size=(2, 2, 1, 200, 128))
    V[0, 0, 198, 5] = np.nan
    V[0, 0, 199, 77] = np.inf
    K[1, 0, 198 - t // 2, 3] = np.nan
    p.write(K, V, [0, 0])
    Q = p.rng.normal(size=(2, G, t, 128))
    O, lse, ref = attend(p, Q, [200, 200], causal=True)
    compare(O, lse, ref, 128)
    for b, first in ((0, 198), (1, 198 - t // 2)):                            # the first position that sees a NaN
        there = np.isnan(ref["O"][b]).any(-1)
        assert there[:, max(0, first - 200 + t):].all() and not there[:, :max(0, first - 200 + t)].any()
    compare(*attend(p, Q, [198, 198 - t // 2], causal=False), 128)            # behind the length: seen by nobody


@pytest.mark.parametrize("d,t,G", [(64, 1, 8), (128, 3, 1), (64, 40, 1), (128, 1, 70)])
def test_few_rows_of_a_long_cache(d, t, G):
    """One key/value head, so that the key axis falls into as many parts as there ever are; a NaN in one of them."""
    p = Pair(1, 1, d, 64, 480)
    K = video_like(p.rng, 1, 1, 30001, d)
    V = p.rng.normal(size=K.shape)
    V[0, 0, 30000, 5] = np.nan
    p.write(K, V, [0])
    Q = p.rng.normal(size=(1, G, t, d)) * 0.3
    compare(*attend(p, Q, [30000], causal=True), d)
    O, lse, ref = attend(p, Q, [30001], causal=True)
    assert np.isnan(ref["O"][0, :, -1]).any(-1).all()
    compare(O, lse, ref, d)


def test_blocks_of_very_different_size():
    """Scales from 2^-40 to 2^40 in one row, and rows that attend to the smallest values alone."""
    p = Pair(1, 1, 64, 64, 8)
    K = p.rng.normal(size=(1, 1, 512, 64)) * 0.1
    V = p.rng.normal(size=(1, 1, 512, 64))
    V *= np.repeat(2.0 ** np.array([0, -40, 3, 40, -2, 20, -20, 1]), 64).reshape(1, 1, 512, 1)
    K[0, 0, :, 0] = np.repeat(np.arange(8.0), 64) * 4
    p.write(K, V, [0])
    Q = p.rng.normal(size=(1, 1, 3, 64)) * 0.1
    Q[0, 0, 1] = 0
    for lists in (None, {(0, 0, 0): [1]}, {(0, 0, 0): [1, 6]}, {(0, 0, 0): [2, 0, 7]}):
        compare(*attend(p, Q, [512], lists=lists, group=3 if lists else 0), 64)


def test_scores_far_from_zero():
    """Rows whose scores are all very low, very high, or rise along the keys by hundreds; an explicit scale."""
    p = Pair(1, 1, 128, 64, 6)
    K = p.rng.normal(size=(1, 1, 384, 128))
    K[0, 0, :, 0] = np.arange(384) * 0.5
    p.write(K, p.rng.normal(size=K.shape), [0])
    Q = p.rng.normal(size=(1, 1, 6, 128))
    Q[0, 0, :, 0] = [0, 40, -40, 3, -3, 100]
    for scale in (0.0, 0.01, 1.0):
        compare(*attend(p, Q, [384], scale=scale, causal=scale == 1.0), 128)


KINDS = [(64, 1, 1), (128, 3, 8), (64, 40, 1), (128, 130, 1)]     # d, t, heads: tiles of 16 and 32 rows, of 64 and 128


def one_channel(p, scores, values, Q0, d, G, t):
    """Into an empty cache keys of one channel, `scores` [n], and `values` [n, d]; queries of about `Q0` in that channel."""
    n = len(scores)
    K = np.zeros((1, 1, n, d))
    K[0, 0, :, 0] = scores
    p.write(K, values.reshape(1, 1, n, d), [0])
    Q = np.zeros((1, G, t, d))
    Q[..., 0] = Q0 * np.linspace(0.98, 1.02, G * t).reshape(1, G, t)
    return Q


@pytest.mark.parametrize("d,t,G", KINDS)
def test_the_smallest_keys(d, t, G):
    """Keys of 2^-126 and more, queries of 2^123: the scale of the keys times that of the scores is below 2^-126."""
    p = Pair(1, 1, d, 64, 3)
    n = 150
    s = p.rng.integers(-15, 16, size=n) * 2.0 ** -126
    Q = one_channel(p, s, p.rng.normal(size=(n, d)), 2.0 ** 123, d, G, t)
    compare(*attend(p, Q, [n]), d)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("first", [True, False])
def test_small_weights_of_zero_values_count(first, d, t, G, ws):
    """Blocks whose values are all zero hold two thirds of the softmax in weights of 2^-10, beside one with values of 2^90: their exponent
    is 208 below its own."""
    p = Pair(1, 1, d, 64, 40)
    n = 40 * 64
    s = np.full(n, -1.0)
    v = np.zeros((n, d))
    own = slice(0, 64) if first else slice(n - 64, n)
    s[own] = -2.0
    s[own.start] = 0.0
    v[own] = p.rng.normal(size=(64, d)) * 2.0 ** 90
    Q = one_channel(p, s, v, 10 * np.log(2), d, G, t)
    compare(*attend(p, Q, [n], scale=1.0, ws=ws), d)


@pytest.mark.parametrize("by", [30, 90, 110])
@pytest.mark.parametrize("d,t,G", KINDS)
def test_large_values_without_weight(d, t, G, by):
    """Values 2^by times larger in the first, a middle and the last block, whose weights are e^-700 and less."""
    for where in ([0], [5], [12], [0, 5, 12]):
        p = Pair(1, 1, d, 64, 13)
        n = 13 * 64
        s = p.rng.integers(-8, 9, size=n) / 8.0
        v = p.rng.normal(size=(n, d))
        far = np.isin(np.arange(n) // 64, where)
        s[far] = -240.0
        v[far] *= 2.0 ** by
        Q = one_channel(p, s, v, 3.0, d, G, t)
        for ws in (True, False):
            compare(*attend(p, Q, [n], scale=1.0, ws=ws), d)


@pytest.mark.parametrize("by", [-110, -40, 40, 110, 200])
@pytest.mark.parametrize("d,t,G", [(64, 70, 1), (128, 130, 1), (128, 8, 4), (64, 12, 1)])
def test_rows_before_a_block_of_another_size(d, t, G, by):
    """Causal rows on both sides of the border of a block whose values are 2^by times those before it: the rows of one tile hold outputs
    of very different size."""
    p = Pair(1, 1, d, 64, 7)
    n = 6 * 64 + t // 2
    K = p.rng.normal(size=(1, 1, n, d))
    V = p.rng.normal(size=K.shape) * 2.0 ** (-100 if by > 120 else 0)
    V[0, 0, 6 * 64:] *= 2.0 ** by
    p.write(K, V, [0])
    Q = p.rng.normal(size=(1, G, t, d))
    for ws in (True, False):
        compare(*attend(p, Q, [n], causal=True, ws=ws), d)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,t,G", KINDS)
def test_many_small_weights_beside_a_block_of_large_values(d, t, G, ws):
    """One key has the weight 1, 4000 have some 2^-17 each and make up the first half of the channels alone; blocks of values 2^8 times
    larger stand between them with no weight to speak of (2^-68)."""
    p = Pair(1, 1, d, 64, 64)
    n = 64 * 64
    s = np.full(n, -1.0)
    v = np.ones((n, d))
    out = np.arange(n) // 64 % 16 < 4
    s[out] = -4.0
    v[out] *= 2.0 ** 8
    s[300] = 0.0                                                               # the dominant key (block 4)
    v[300, :d // 2] = 0
    Q = one_channel(p, s, v, 17 * np.log(2), d, G, t)
    compare(*attend(p, Q, [n], scale=1.0, ws=ws), d)


@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("size", [2.0 ** 19, 2.0 ** 22, 2.0 ** 24, 2.0 ** 26, 2.0 ** 60, 2.0 ** 110])
def test_scores_of_many_millions(size, d, t, G):
    """Scores whose neighbours in 32 bits are from 1/2 apart on, rising along the keys, under values of different scales: the bound leaves the
    weights open there, but an output is a mean of the values."""
    p = Pair(1, 1, d, 64, 12)
    n = 12 * 64
    s = np.sort(p.rng.integers(-15, 16, size=n) / 1.0)
    v = p.rng.uniform(1, 2, size=(n, d)) * np.repeat(2.0 ** p.rng.integers(0, 8, size=12), 64)[:, None]
    Q = one_channel(p, s, v, size, d, G, t)
    for sign in (1, -1):
        O, lse, ref = attend(p, Q * sign, [n], scale=1.0)
        compare(O, lse, ref, d)
        assert O.min() >= 1 and O.max() <= 256


@pytest.mark.parametrize("by", [20, 60, 76])
@pytest.mark.parametrize("d,t,G", KINDS)
def test_channels_that_only_the_small_blocks_fill(d, t, G, by):
    """Every block has weight; values 2^by times larger stand in every fourth one and leave the first half of the channels zero, which the
    others make up alone."""
    for shift in (0, 3):
        p = Pair(1, 1, d, 64, 16)
        n = 16 * 64
        s = p.rng.integers(-8, 9, size=n) / 8.0
        v = p.rng.uniform(1, 2, size=(n, d))
        far = (np.arange(n) // 64 + shift) % 4 == 0
        v[far] *= 2.0 ** by
        v[far, :d // 2] = 0
        Q = one_channel(p, s, v, 1.0, d, G, t)
        for ws in (True, False):
            compare(*attend(p, Q, [n], scale=1.0, ws=ws), d)



def test_offsets_past_32_bits():
    """The same tokens in the first and in the last pages of a pool of more than 4 GiB of codes for K alone."""
    pages, hk, d, block = 33000, 8, 128, 128
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 10 GB")
    gpu = rb.allocate_cache(2, hk, d, block, pages, 3, DEV)
    assert gpu.k_codes.numel() > 1 << 32
    gpu.table.copy_(torch.tensor([[1, 0, 2], [pages - 1, pages - 3, pages - 2]]))
    rng = np.random.default_rng(0)
    K, V = (bf16(np.repeat(rng.normal(size=(1, hk, 300, d)), 2, axis=0)) for _ in range(2))
    rb.rsa_cache_write(gpu, rb.make_rows(K), K, V, i32([0, 0]))
    R, S = torch.zeros_like(K), torch.zeros_like(V)
    rb.rsa_cache_read(gpu, rb.make_rows(K), i32([0, 0]), None, R, S)
    assert torch.equal(R[0], R[1]) and torch.equal(S[0], S[1]) and (R - K).abs().max() <= 2.0 ** -4 * K.abs().max()
    Q = bf16(np.repeat(rng.normal(size=(1, hk, 5, d)), 2, axis=0))
    O, rows = torch.zeros_like(Q), rb.make_rows(Q)
    idx, kept = torch.zeros(2, hk, 1, 3, dtype=torch.int32, device=DEV), torch.zeros(2, hk, 1, dtype=torch.int32, device=DEV)
    rb.rsa_cache_select(gpu, rows, Q, i32([300, 300]), None, 5, 2, 0, 1, 0, idx, kept)
    rb.rsa_cache_attn(gpu, rows, Q, i32([300, 300]), None, 0.0, 0, idx, kept, 5, O)
    assert torch.equal(O[0], O[1]) and O.abs().max() > 0 and torch.equal(idx[0], idx[1])


def pool(batch, hk, d, block, max_blocks, pages, seed=0):
    """A Pair whose sequences take their blocks from the same few written pages (nothing is written through it afterwards)."""
    p = Pair(batch, hk, d, block, max_blocks, seed, np.random.default_rng(seed + 1).integers(0, pages, size=(batch, max_blocks)), pages)
    one = Pair(1, hk, d, block, pages, seed + 2, np.arange(pages).reshape(1, pages), pages)
    one.gpu = rb.cache_of(p.gpu.k_codes, p.gpu.v_codes, p.gpu.scales, p.gpu.k_mean, one.gpu.table, block)
    one.fill([pages * block], spread=0.5)
    p.ref.held = one.ref.held
    return p


# ---- many rows, long tables ----------------------------------------------------------------------
@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,batch,hk,G,t,blocks,keep", [
    (128, 3, 2, 2, 1, 1025, 100), (64, 3, 1, 1, 2, 2000, 150), (128, 2, 2, 1, 26, 1500, 40), (64, 2, 3, 2, 20, 4096, 64), (64, 3, 1, 4, 1, 4097, 300),
    (128, 1, 1, 1, 3, 9000, 2000), (64, 2, 1, 1, 2, 16384, 64)])
def test_select_from_long_tables(d, batch, hk, G, t, blocks, keep, ws):
    """Every form of the choice, several sequences of different length, means and scales drawn directly."""
    p = Pair(batch, hk, d, 64, blocks, table=np.random.default_rng(5).integers(-3, 200, size=(batch, blocks)), pages=200)
    for page in range(200):
        for h in range(hk):
            q = p.ref.held.setdefault((page, h), co.Page(64, d))
            q.mean, q.em = p.rng.integers(-127, 128, size=d), int(p.rng.integers(-9, -5))
    p.gpu.k_mean.copy_(torch.as_tensor(np.array([[p.ref.held[i, h].mean for h in range(hk)] for i in range(200)])))
    p.gpu.scales.copy_(torch.as_tensor(np.array([[[1, 1, 2.0 ** p.ref.held[i, h].em, 0] for h in range(hk)] for i in range(200)])))
    lens = [blocks * 64 - i * (blocks * 64 // 3) for i in range(batch)]
    select(p, p.rng.normal(size=(batch, hk * G, t, d)), lens, [max(1, t - i) for i in range(batch)], 1, keep, 1, 2, True, ws=ws)


def test_attention_in_several_rounds_of_workgroups():
    """76 rows on up to 6400 keys, each in parts, more workgroups than the chip takes at once."""
    p = pool(19, 4, 128, 64, 100, 30)
    lens = [6400 - 300 * i for i in range(19)]
    compare(*attend(p, p.rng.normal(size=(19, 8, 1, 128)), lens, causal=True), 128)


@pytest.mark.parametrize("d,t,G", [(64, 140, 1), (128, 75, 2)])
def test_prompts_of_many_tiles(d, t, G):
    """528 tiles of causal prompts, so that those of a sequence's last tokens go first: the same bits as a few sequences at a time."""
    batch = 33
    p = pool(batch, 8, d, 64, 3, 20)
    lens, q_len = [t + i for i in range(batch)], [t - i % 5 for i in range(batch)]
    Q = bf16(p.rng.normal(size=(batch, 8 * G, t, d)))
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:3], 7.0, device=DEV)
    rb.rsa_cache_attn(p.gpu, rb.make_rows(Q), Q, i32(lens), i32(q_len), 0.0, rb.RSA_CACHE_CAUSAL, None, None, 0, O, lse)
    for at in range(0, batch, 11):
        part = Pair(11, 8, d, 64, 3, table=p.ref.table[at:at + 11], pages=20)
        part.gpu = rb.cache_of(p.gpu.k_codes, p.gpu.v_codes, p.gpu.scales, p.gpu.k_mean, part.gpu.table, 64)
        q, o, own = Q[at:at + 11], torch.full_like(Q[at:at + 11], 7.0), torch.full((11, 8 * G, t), 7.0, device=DEV)
        rb.rsa_cache_attn(part.gpu, rb.make_rows(q), q, i32(lens[at:at + 11]), i32(q_len[at:at + 11]), 0.0, rb.RSA_CACHE_CAUSAL, None, None, 0, o, own)
        assert torch.equal(O[at:at + 11].view(torch.int16), o.view(torch.int16)) and torch.equal(lse[at:at + 11], own)
    few = slice(16, 18)
    p.ref.table = p.ref.table[few]
    compare(f64(O[few]), lse[few].cpu().double().numpy(), p.ref.attend(f64(Q[few]), lens[few], q_len[few], 0.0, True), d)


# ---- together ------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,block,G,steps", [(128, 64, 2, [100, 1, 1, 5, 70, 1]), (64, 128, 1, [130, 128, 3, 1])])
def test_a_sequence_step_by_step(d, block, G, steps):
    """Prompt, tokens, drafts and chunks through cached_sparse_attention: lists exact, outputs within the bound."""
    p = Pair(2, 2, d, block, 5)
    lens = np.zeros(2, dtype=int)
    for t in steps:
        r = [t, max(1, t - 1)]
        lens += r
        K, V, Q = (video_like(p.rng, 2, h, t, d) for h in (2, 2, 2 * G))
        Kd, Vd, Qd = bf16(K), bf16(V), bf16(Q)
        p.ref.write(f64(Kd), f64(Vd), (lens - r).tolist(), r)
        group, keep = (1 if t <= 8 else 16), 2
        groups = -(-t // group)
        idx = torch.zeros(2, 2, groups, 4, dtype=torch.int32, device=DEV)
        kept = torch.zeros(2, 2, groups, dtype=torch.int32, device=DEV)
        O, lse = torch.full_like(Qd, 7.0), torch.full(Qd.shape[:3], 7.0, device=DEV)
        ws = torch.empty(max(256, *rb.rsa_cache_workspace_bytes(p.gpu, rb.make_rows(Qd), group)), dtype=torch.uint8, device=DEV)
        rb.cached_sparse_attention(p.gpu, Kd, Vd, Qd, O, i32(lens), i32(r), group, keep, idx, kept, lse=lse, ws=ws)
        want = p.ref.select(f64(Qd), lens, r, group, keep, 1, 1, True)
        for (b, h, g), x in want.items():
            assert idx[b, h, g, :int(kept[b, h, g])].tolist() == x
        compare(f64(O), lse.cpu().double().numpy(), p.ref.attend(f64(Qd), lens, r, 0.0, True, want, group), d)
        p.check_pages()


def test_a_step_with_more_queries_than_rows():
    """A q_len beyond the rows counts as all of them, for where the keys go as for the queries' positions."""
    p = Pair(2, 1, 64, 64, 3)
    p.fill([70, 9])
    K, V, Q = (video_like(p.rng, 2, h, 3, 64) for h in (1, 1, 2))
    Kd, Vd, Qd = bf16(K), bf16(V), bf16(Q)
    lens, r = [73, 11], [99, 2]
    p.ref.write(f64(Kd), f64(Vd), [70, 9], [3, 2])
    idx, kept = torch.zeros(2, 1, 3, 4, dtype=torch.int32, device=DEV), torch.zeros(2, 1, 3, dtype=torch.int32, device=DEV)
    O, lse = torch.full_like(Qd, 7.0), torch.full(Qd.shape[:3], 7.0, device=DEV)
    rb.cached_sparse_attention(p.gpu, Kd, Vd, Qd, O, i32(lens), i32(r), 1, 2, idx, kept, lse=lse)
    want = p.ref.select(f64(Qd), lens, [3, 2], 1, 2, 1, 1, True)
    compare(f64(O), lse.cpu().double().numpy(), p.ref.attend(f64(Qd), lens, [3, 2], 0.0, True, want, 1), 64)
    p.check_pages()
    with pytest.raises(ValueError):
        rb.cached_sparse_attention(p.gpu, Kd[:, :, :2], Vd[:, :, :2], Qd, O, i32(lens), None, 1, 2, idx, kept)


def test_on_another_stream_and_replayed():
    """The three calls on a stream of their own, and captured into a graph that is replayed with new contents in between eager work."""
    p = Pair(2, 2, 128, 64, 6)
    p.fill([200, 150])
    Qn = [video_like(p.rng, 2, 4, 1, 128) for _ in range(4)]
    Kn = [video_like(p.rng, 2, 2, 1, 128) for _ in range(4)]
    Q, K, V = bf16(Qn[0]), bf16(Kn[0]), bf16(Kn[0])
    O, lse = torch.zeros_like(Q), torch.zeros(2, 4, 1, device=DEV)
    idx, kept = torch.zeros(2, 2, 1, 4, dtype=torch.int32, device=DEV), torch.zeros(2, 2, 1, dtype=torch.int32, device=DEV)
    kv_len = i32([200, 150])
    ws = torch.empty(max(256, *rb.rsa_cache_workspace_bytes(p.gpu, rb.make_rows(Q), 1)), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        rb.cached_sparse_attention(p.gpu, K, V, Q, O, kv_len, None, 1, 3, idx, kept, lse=lse, ws=ws, stream=stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    lens = np.array([200, 150])
    for i in range(4):
        Q.copy_(bf16(Qn[i])); K.copy_(bf16(Kn[i])); V.copy_(bf16(Kn[i] * 0.5))
        kv_len += 1
        lens += 1
        torch.cuda.synchronize()
        if i == 0:
            step(side)
        else:
            if i == 1:
                with torch.cuda.graph(graph):
                    step()
            graph.replay()
        torch.cuda.synchronize()
        p.ref.write(f64(K), f64(V), (lens - 1).tolist())
        want = p.ref.select(f64(Q), lens, None, 1, 3, 1, 1, True)
        compare(f64(O), lse.cpu().double().numpy(), p.ref.attend(f64(Q), lens, None, 0.0, True, want, 1), 128)
        eager = torch.zeros_like(O)
        rb.rsa_cache_attn(p.gpu, rb.make_rows(Q), Q, kv_len, None, 0.0, 1, idx, kept, 1, eager, None, ws)
        assert torch.equal(eager, O)
    p.check_pages()


def test_the_same_call_twice_gives_the_same_bits():
    p = Pair(3, 2, 128, 128, 10)
    p.fill([1200, 700, 1280])
    Q = bf16(video_like(p.rng, 3, 4, 2, 128))
    rows, kv = rb.make_rows(Q), i32([1200, 700, 1280])
    ws = torch.empty(rb.rsa_cache_workspace_bytes(p.gpu, rows, 0)[1], dtype=torch.uint8, device=DEV)
    got = []
    for _ in range(3):
        O = torch.empty_like(Q)
        rb.rsa_cache_attn(p.gpu, rows, Q, kv, None, 0.0, 1, None, None, 0, O, None, ws)
        got.append(O.view(torch.int16).clone())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    O = Q.clone()                                                   # O may be Q
    rb.rsa_cache_attn(p.gpu, rows, O, kv, None, 0.0, 1, None, None, 0, O, None, ws)
    assert torch.equal(O.view(torch.int16), got[0])


# ---- refusals of the binding ---------------------------------------------------------------------
def test_binding_refusals():
    p = Pair(2, 2, 64, 64, 4)
    K = bf16(np.zeros((2, 2, 3, 64)))
    rows, kv = rb.make_rows(K), i32([3, 3])
    for bad in (K.float(), K[:1], K[:, :, :2], bf16(np.zeros((2, 2, 3, 64)), "bthd"), K.cpu()):
        with pytest.raises(ValueError):
            rb.rsa_cache_write(p.gpu, rows, bad, K, kv)
    for bad in (kv.long(), kv[:1], kv.cpu(), i32([1, 2, 3, 4])[::2]):
        with pytest.raises(ValueError):
            rb.rsa_cache_write(p.gpu, rows, K, K, bad)
    idx, kept = torch.zeros(2, 2, 3, 2, dtype=torch.int32, device=DEV), torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    for a, b in ((idx.long(), kept), (idx[:, :, :2], kept), (idx, kept.float()), (idx, kept[:, :1]), (idx.transpose(2, 3), kept)):
        with pytest.raises(ValueError):
            rb.rsa_cache_attn(p.gpu, rows, K, kv, None, 0.0, 0, a, b, 1, torch.empty_like(K))
    with pytest.raises(ValueError):
        rb.rsa_cache_attn(p.gpu, rows, K, kv, None, 0.0, 0, None, None, 0, torch.empty_like(K), torch.zeros(2, 2, 4, device=DEV))
    with pytest.raises(rb.RsaError) as e:
        rb.rsa_cache_select(p.gpu, rows, K, kv, None, 1, 4, 0, 1, 0, idx, kept)
    assert e.value.status == -5                                     # lists of 2 entries for keep = 4
    with pytest.raises(rb.RsaError) as e:
        rb.rsa_cache_attn(p.gpu, rows, K, kv, None, 0.0, 0, None, None, 0, torch.empty_like(K), None, torch.zeros(1024, dtype=torch.uint8, device=DEV)[8:])
    assert e.value.status == -4                                     # not on a boundary of 256 bytes
    with pytest.raises(rb.RsaError) as e:
        rb.rsa_cache_attn(p.gpu, rows, K, kv, None, 0.0, 0, idx, None, 1, torch.empty_like(K))
    assert e.value.status == -1
