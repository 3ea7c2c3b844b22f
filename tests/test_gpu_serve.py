"""The 4-bit cache, page assignment and rotary positions on the GPU against their oracle (oracle/serve_oracle.py).

What a write leaves, what is read back, the means behind the selection, tables, positions and slots are exact. Outputs of the attention are
held to a bound made of its roundings, for each element, with A = sum p |v| / sum p over the same keys:

  |O - O64| <= 2^-8 |O64|                       the output in bf16: half a step
             + (2^-8 + 2 e_s + 4 n 2^-24) A     a weight times its token's scale in bf16: half a step; scores off by e_s change p by e_s of
                                                itself, above and below the division; sums of n terms in 32 bits, each way
             + n 2^-126                         products below the smallest normal number may vanish
  e_s = (d + 16) 2^-24 max_j sum|q||k_j| * scale   the dot product in 32 bits and the few operations behind it
  |lse - lse64| <= 2 e_s + 4 n 2^-24 + 2^-21 max(1, |lse|)

Rotary: y = f (x1 c - x2 s) with c and s within 2^-22 (series 2^-25, its argument in 32 bits 2^-24, roundings), two products and a sum in 32
bits, one rounding to bf16: |y - y64| <= 2^-8 |y64| + 2^-21 f (|x1| + |x2|).
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import serve_oracle as so
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
    b, h, t, d = shape
    x = rng.normal(size=shape) * 0.6 + np.cumsum(rng.normal(size=shape), axis=2) * 0.15
    return x * np.exp(rng.normal(size=(b, h, t, 1)) * spread)


def places(block, d):
    """Half bytes of (token, channel) in a page's keys and values; bytes of the keys' exponents, 16-bit places of the values' scales."""
    t, ch = np.arange(block)[:, None], np.arange(d)[None]
    u = t % 64
    k = t // 64 * (68 * d) + ((u // 16 * (d // 32) + ch // 32) * 16 + u % 16) * 32 + ch % 32
    ks = t // 64 * (34 * d) + 32 * d + (ch // 32 * 16 + u % 16) * 4 + u // 16
    v = t // 64 * (64 * d + 256) + ((ch // 32 * 4 + u % 16 // 4) * 16 + ch % 16) * 32 + ch % 32 // 16 * 16 + u // 16 * 4 + u % 4
    vs = t[:, 0] // 64 * (16 * d + 64) + 16 * d + u[:, 0] % 16 // 4 * 16 + u[:, 0] // 16 * 4 + u[:, 0] % 4
    return k, ks, v, vs


class Pair:
    """A 4-bit cache on the GPU and the oracle's, with the same table; pages that were not written hold 0xff everywhere."""

    width = 0          # entries of a row of the table at least, the last ones empty (more than 32 rows are taken otherwise on a short one)

    def __init__(self, batch, hk, d, block, max_blocks, seed=0, table=None, pages=None):
        n = batch * max_blocks
        self.rng = np.random.default_rng(seed)
        if table is None:
            pages = pages or n + 2
            table = self.rng.permutation(pages)[:n].reshape(batch, max_blocks)
        if max_blocks < self.width:
            table = np.concatenate([np.asarray(table), np.full((batch, self.width - max_blocks), -1)], axis=1)
            max_blocks = self.width
        self.gpu = rb.allocate_cache(batch, hk, d, block, pages, max_blocks, DEV, bits=4)
        self.gpu.k_codes.fill_(0xff)
        self.gpu.v_codes.fill_(0xff)
        self.gpu.scales.fill_(float("nan"))
        self.gpu.k_mean.fill_(77)
        self.gpu.table.copy_(torch.as_tensor(np.asarray(table, dtype=np.int32)))
        self.ref = so.Cache(hk, d, block, table, pages)
        self.written = {}                                  # (page, head) -> tokens that were ever written
        self.batch, self.hk, self.d, self.block = batch, hk, d, block

    def write(self, K, V, start, count=None, layout="bhtd", stream=None):
        K, V = bf16(K, layout), bf16(V, layout)
        rb.rsa_fourbit_write(self.gpu, rb.make_rows(K), K, V, i32(start), i32(count), stream)
        self.ref.write(f64(K), f64(V), start, count)
        t = K.shape[2]
        for b in range(self.batch):
            n = t if count is None else min(count[b], t)
            for tok in range(start[b], start[b] + n) if start[b] >= 0 else ():
                page = self.ref.page_of(b, tok // self.block)
                if page >= 0:
                    self.written.setdefault(page, np.zeros(self.block, dtype=bool))[tok % self.block] = True

    def fill(self, lens, spread=0.0):
        t = max(max(lens), 1)
        K = video_like(self.rng, self.batch, self.hk, t, self.d, spread=spread)
        self.write(K, self.rng.normal(size=K.shape) * np.exp(self.rng.normal(size=K.shape[:3] + (1,)) * spread), [0] * self.batch, lens)

    def check_pages(self):
        """Codes and scales of every token, bit for bit; nothing else touched."""
        scales, mean = self.gpu.scales.cpu().numpy(), self.gpu.k_mean.cpu().numpy()
        k, ks, v, vs = places(self.block, self.d)
        kc, vc = self.gpu.k_codes.cpu().numpy(), self.gpu.v_codes.cpu().numpy()
        levels = np.concatenate([so.LEVELS, -so.LEVELS])
        for page in range(scales.shape[0]):
            for h in range(self.hk):
                p = self.ref.held.get((page, h))
                if p is None:
                    assert np.isnan(scales[page, h]).all() and (mean[page, h] == 77).all() and (kc[page, h] == 255).all() and (vc[page, h] == 255).all()
                    continue
                there = self.written[page]
                code_k, code_v = kc[page, h][k // 2] >> (k % 2 * 4) & 15, vc[page, h][v // 2] >> (v % 2 * 4) & 15
                e, s = kc[page, h][ks].astype(int) - 127, vc[page, h].view(np.uint16)[vs].astype(np.uint32) << 16
                with np.errstate(over="ignore", invalid="ignore"):
                    got_k = np.where(e == 128, np.nan, levels[code_k] * np.exp2(e.astype(float)))
                    got_v = levels[code_v] * s.view(np.float32).astype(np.float64)[:, None]
                got_k, got_v = (np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x) for x in (got_k, got_v))
                np.testing.assert_array_equal(got_k[there], p.k[there])
                np.testing.assert_array_equal(got_v[there], p.v[there])
                assert (code_k[~there] == 15).all() and (code_v[~there] == 15).all() and (e[~there] == 128).all() and (s[~there] == 0xffff0000).all()
                np.testing.assert_array_equal(mean[page, h], p.mean)
                assert scales[page, h].tolist() == [0.0, 0.0, 2.0 ** p.em, 0.0]


@pytest.fixture
def wide(request):
    Pair.width = 20 if request.param else 0
    yield
    Pair.width = 0


WIDE = pytest.mark.parametrize("wide", [False, True], indirect=True)


def attend(pair, Q, kv_len, q_len=None, scale=0.0, causal=False, lists=None, group=0, layout="bhtd", ws=True, stream=None, list_len=0):
    """rsa_fourbit_attn on Q (numpy) -> (outputs, lse) as numpy, and the oracle's."""
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
        n = rb.rsa_fourbit_workspace_bytes(pair.gpu, rows, group)
        scratch = torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device=DEV)     # NaN wherever it is read before it is written
    rb.rsa_fourbit_attn(pair.gpu, rows, Qd, i32(kv_len), i32(q_len), scale, rb.RSA_CACHE_CAUSAL if causal else 0, idx, kept, group, O, lse, scratch, stream)
    torch.cuda.synchronize()
    ref = pair.ref.attend(f64(Qd), kv_len, q_len, scale, causal, lists, group)
    few = (min(group, Q.shape[2]) if lists is not None else Q.shape[2]) * (Q.shape[1] // pair.hk) <= 32
    return f64(O), lse.cpu().double().numpy(), {**ref, "P": 2.0 ** -15 if few else 2.0 ** -8}


def compare(O, lse, ref, d):
    """Weights are rounded by half a step of bf16, 2^-8 of them, and an output is off by at most that of A = sum p |v| / sum p. Up to 32 rows: they are cut to
    bf16, which leaves less than 2^-7 of a weight, and that is rounded to bf16 in turn: 2^-15. What vanishes: a weight times its token's scale below
    2^-126, and a weight below 2^-133 under a scale of at most 2^7, both times a code of at most 6: 6 * 2^-126 for each key."""
    isq = ref["isq"]
    assert (O[~isq] == 7.0).all() and (lse[~isq] == 7.0).all(), "rows behind the last query were written"
    O, lse = O[isq], lse[isq]
    want, A, want_lse, S, n = (ref[k][isq] for k in ("O", "A", "lse", "S", "n"))
    empty = n == 0
    assert (O[empty] == 0).all() and np.isneginf(lse[empty]).all()
    O, lse, want, A, want_lse, S, n = (x[~empty] for x in (O, lse, want, A, want_lse, S, n))
    assert np.array_equal(np.isnan(O), np.isnan(want)) and np.array_equal(np.isnan(lse), np.isnan(want_lse))
    es = (d + 16) * 2.0 ** -24 * S
    bound = 2.0 ** -8 * np.abs(want) + (ref.get("P", 2.0 ** -8) + 2 * es + 4 * n * 2.0 ** -24)[:, None] * A + n[:, None] * 6 * 2.0 ** -126
    ok = ~np.isnan(want)
    worst = (np.abs(O - want)[ok] / bound[ok]).max(initial=0)
    fine = ~np.isnan(want_lse)
    lb = 2 * es + 4 * n * 2.0 ** -24 + 2.0 ** -21 * np.maximum(1, np.abs(np.where(fine, want_lse, 0)))
    worst_lse = (np.abs(lse - want_lse)[fine] / lb[fine]).max(initial=0)
    print(f"of the bound: outputs {worst:.2f}, lse {worst_lse:.2f}")
    assert worst <= 1 and worst_lse <= 1


# ---- writing and reading -------------------------------------------------------------------------
SIZES = [(64, 64, "bhtd"), (64, 128, "bthd"), (128, 64, "bthd"), (128, 128, "bhtd")]


@pytest.mark.parametrize("d,block,layout", SIZES)
def test_write_in_pieces(d, block, layout):
    """Ragged pieces: inside a block, across several, one token, none, more than there are rows, back to an earlier length."""
    p = Pair(3, 2, d, block, 6)
    pos = np.zeros(3, dtype=int)
    for step, (t, count) in enumerate([(5, [5, 1, 0]), (1, [1, 1, 1]), (200, [200, 3, 131]), (block, None), (70, [64, -3, 99]), (2, [2, 2, 2])]):
        K = video_like(p.rng, 3, 2, t, d, spread=1.0)
        p.write(K, p.rng.normal(size=K.shape) * 2.0 ** (3 - step), pos.tolist(), count, layout)
        pos += np.clip(count if count is not None else [t] * 3, 0, t)
        p.check_pages()
    p.write(video_like(p.rng, 3, 2, 9, d), video_like(p.rng, 3, 2, 9, d), [-1, 30, block + 2], None, layout)
    p.check_pages()


@pytest.mark.parametrize("d,block", [(64, 64), (128, 128), (128, 64), (64, 128)])
def test_token_by_token(d, block):
    p = Pair(2, 1, d, block, 2)
    K = video_like(p.rng, 2, 1, block + 5, d, spread=2.0)
    V = p.rng.normal(size=K.shape) * np.exp(p.rng.normal(size=(2, 1, block + 5, 1)) * 2)
    for t in range(block + 5):
        p.write(K[:, :, t:t + 1], V[:, :, t:t + 1], [t, t])
    p.check_pages()
    q = Pair(2, 1, d, block, 2)
    q.write(K, V, [0, 0])
    q.check_pages()
    for a, b in zip((p.gpu.k_codes, p.gpu.v_codes, p.gpu.k_mean, p.gpu.scales[..., 2]), (q.gpu.k_codes, q.gpu.v_codes, q.gpu.k_mean, q.gpu.scales[..., 2])):
        assert torch.equal(torch.nan_to_num(a) if a.is_floating_point() else a, torch.nan_to_num(b) if b.is_floating_point() else b)


@pytest.mark.parametrize("d,block", [(64, 64), (128, 128)])
def test_write_at_the_ends_of_the_range(d, block):
    """Zeros, the smallest and largest bf16, infinities, NaN, every boundary between codes, values that halve down a row."""
    p = Pair(1, 1, d, block, 8 * 64 // block)
    edge = np.zeros((1, 1, 8 * 64, d))
    edge[0, 0, 64:128] = np.ldexp(p.rng.normal(size=(64, d)), -p.rng.integers(120, 136, size=(64, 1)))
    edge[0, 0, 128:192] = np.ldexp((1.0 + p.rng.integers(0, 128, size=(64, d)) / 128) * p.rng.choice([-1, 1], size=(64, d)), 127)
    edge[0, 0, 192:256] = p.rng.normal(size=(64, d))
    edge[0, 0, 200, 3], edge[0, 0, 201, 40], edge[0, 0, 202, 35] = np.inf, -np.inf, np.nan
    edge[0, 0, 256:320] = np.nan
    edge[0, 0, 320:384] = np.linspace(-6, 6, 64 * d).reshape(64, d)
    edge[0, 0, 384:448] = p.rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5], size=(64, d))
    edge[0, 0, 448:] = np.ldexp(1.5 + p.rng.integers(0, 3, size=(64, 1)) / 128 - 1 / 128, -np.arange(d) % 40)
    x = torch.as_tensor(edge).float()
    x = torch.where(torch.isfinite(x), x.clamp(-3.3895313892515355e38, 3.3895313892515355e38), x)
    p.write(x.numpy(), x.flip(2).numpy(), [0])
    p.check_pages()
    R, S = bf16(np.zeros((1, 1, 512, d))), bf16(np.zeros((1, 1, 512, d)))
    rb.rsa_fourbit_read(p.gpu, rb.make_rows(R), i32([0]), None, R, S)
    k, v, _ = p.ref.rows(0, 0, 0, 512)
    np.testing.assert_array_equal(f64(R)[0, 0], k)
    np.testing.assert_array_equal(f64(S)[0, 0], v)


def test_write_passes_over_what_is_no_page():
    table = [[2, -1, 9, 0], [7, 1, 3, -5]]                      # pages 0..3 exist
    p = Pair(2, 2, 64, 64, 4, table=table, pages=4)
    K = video_like(p.rng, 2, 2, 300, 64)                        # more than the table holds, too
    p.write(K, K[:, :, ::-1], [0, 30])
    p.check_pages()
    R, S = bf16(np.full((2, 2, 300, 64), 7.0)), bf16(np.full((2, 2, 300, 64), 7.0))
    rb.rsa_fourbit_read(p.gpu, rb.make_rows(R), i32([0, 30]), None, R, S)
    for b, s in enumerate((0, 30)):
        for h in range(2):
            k, v, there = p.ref.rows(b, h, s, s + 300)
            np.testing.assert_array_equal(f64(R)[b, h], np.where(there[:, None], k, 7.0))
            np.testing.assert_array_equal(f64(S)[b, h], np.where(there[:, None], v, 7.0))


@pytest.mark.parametrize("d,block,layout", SIZES)
def test_read_back(d, block, layout):
    p = Pair(3, 2, d, block, 4)
    p.fill([4 * block, 2 * block + 3, 1], spread=1.0)
    t = 2 * block + 9
    for start, count in (([block - 3, 2, 0], [t, 2 * block + 1, 1]), ([5, 1, 0], [2, 3, 0]), ([-1, 0, 0], [1, 1, 1])):
        K, V = bf16(np.full((3, 2, t, d), 7.0), layout), bf16(np.full((3, 2, t, d), 7.0), layout)
        rb.rsa_fourbit_read(p.gpu, rb.make_rows(K), i32(start), i32(count), K, V)
        for b in range(3):
            n = count[b] if start[b] >= 0 else 0
            for h in range(2):
                k, v, _ = p.ref.rows(b, h, start[b], start[b] + n) if n else (np.zeros((0, d)),) * 2 + (None,)
                for got, want in ((K, k), (V, v)):
                    np.testing.assert_array_equal(f64(got)[b, h, :n], want)
                    assert (f64(got)[b, h, n:] == 7.0).all()


@pytest.mark.parametrize("d,block,G,t,group,keep,causal", [(64, 64, 1, 1, 1, 3, True), (128, 128, 4, 1, 1, 5, True), (128, 64, 1, 150, 64, 6, True),
                                                           (64, 128, 2, 131, 50, 2, False)])
def test_select_reads_the_means(d, block, G, t, group, keep, causal):
    p = Pair(3, 2, d, block, 20)
    lens = [20 * block, 11 * block + 7, t]
    p.fill(lens)
    Qd = bf16(video_like(p.rng, 3, 2 * G, t, d))
    groups, n = -(-t // group), min(20, max(keep, 2 + -(-group // block) + 1))
    idx, kept = torch.zeros(3, 2, groups, n, dtype=torch.int32, device=DEV), torch.zeros(3, 2, groups, dtype=torch.int32, device=DEV)
    rb.rsa_cache_select(p.gpu, rb.make_rows(Qd), Qd, i32(lens), None, group, keep, 1, 1, rb.RSA_CACHE_CAUSAL if causal else 0, idx, kept)
    for (b, h, g), x in p.ref.select(f64(Qd), lens, None, group, keep, 1, 1, causal).items():
        assert int(kept[b, h, g]) == len(x) and idx[b, h, g].tolist() == x + [-1] * (n - len(x))


# ---- attention -----------------------------------------------------------------------------------
SHAPES = [  # d, block, G, t, lens, q_len, causal
    (64, 64, 1, 1, [1], None, True),                              # one key
    (64, 64, 1, 1, [65, 1000, 64], None, False),
    (128, 64, 4, 1, [700, 1, 130], None, True),
    (128, 128, 8, 1, [129, 1300, 128], None, True),
    (64, 128, 5, 3, [200, 3, 500], [3, 3, 2], True),              # heads that fill no tile
    (128, 128, 1, 17, [300, 17, 900], [17, 5, 16], True),
    (64, 64, 3, 9, [300, 9, 900], [9, 5, 8], True),
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
    (64, 128, 1, 60, [700, 60, 130], None, True),
    (128, 64, 1, 50, [700, 60, 130], None, True),
]


@WIDE
@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,block,G,t,lens,q_len,causal", SHAPES)
def test_attention(wide, d, block, G, t, lens, q_len, causal, ws):
    b = len(lens)
    p = Pair(b, 2, d, block, -(-max(lens) // block) + 1)
    p.fill(lens, spread=0.5)
    Q = video_like(p.rng, b, 2 * G, t, d)
    compare(*attend(p, Q, lens, q_len, causal=causal, layout="bthd" if t % 2 else "bhtd", ws=ws), d)


@WIDE
@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,block,G,t,group,causal", [(64, 64, 1, 1, 1, True), (128, 64, 4, 1, 1, True), (128, 128, 3, 5, 1, True),
                                                      (128, 128, 1, 200, 128, False), (128, 64, 2, 90, 64, True), (64, 128, 1, 77, 20, True),
                                                      (128, 128, 1, 129, 1 << 30, False)])
def test_attention_over_lists(wide, d, block, G, t, group, causal, ws):
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


@WIDE
def test_attention_passes_over_what_is_no_page(wide):
    table = np.arange(20).reshape(2, 10)
    table[0, 3], table[0, 9], table[1, 0], table[1, 5] = -1, 1000, 77, -3
    p = Pair(2, 2, 128, 64, 10, table=table, pages=20)
    p.fill([640, 500])
    for t in (3, 40):
        Q = p.rng.normal(size=(2, 4, t, 128))
        compare(*attend(p, Q, [640, 500], causal=True), 128)
        compare(*attend(p, Q, [64 * 3 + 1, 30], causal=False), 128)           # the only visible block of the second is missing
        compare(*attend(p, Q, [0, 2], [3, 3], causal=True), 128)              # no token; positions before the first
        compare(*attend(p, Q, [5000, -7], [3, 3], causal=False), 128)         # longer than the table; negative


KINDS = [(64, 1, 1), (128, 1, 4), (128, 5, 4), (64, 40, 1), (128, 50, 1), (128, 70, 2)]


@WIDE
@pytest.mark.parametrize("d,t,G", [(128, 4, 2), (64, 4, 2), (128, 40, 1), (64, 40, 1), (128, 140, 1)])
def test_nan_stays_with_the_rows_that_see_it(wide, d, t, G):
    """NaN among values and among keys of single tokens: causal rows before them are unharmed."""
    p = Pair(2, 1, d, 64, 4)
    K, V = p.rng.normal(size=(2, 2, 1, 200, d))
    V[0, 0, 198, 5] = np.nan
    V[0, 0, 199, 37] = np.inf
    K[1, 0, 198 - t // 2, 3] = np.nan
    p.write(K, V, [0, 0])
    Q = p.rng.normal(size=(2, G, t, d))
    O, lse, ref = attend(p, Q, [200, 200], causal=True)
    compare(O, lse, ref, d)
    for b, first in ((0, 198), (1, 198 - t // 2)):                            # the first position that sees a NaN
        there = np.isnan(ref["O"][b]).any(-1)
        assert there[:, max(0, first - 200 + t):].all() and not there[:, :max(0, first - 200 + t)].any()
    compare(*attend(p, Q, [198, 198 - t // 2], causal=False), d)              # behind the length: seen by nobody


@WIDE
@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("by", [20, 60, 90])
@pytest.mark.parametrize("d,t,G", KINDS)
def test_values_of_very_different_size(wide, d, t, G, by, ws):
    """Every fourth block holds values 2^by times the others' and zeros in half of the channels; then none of its weight."""
    p = Pair(1, 1, d, 64, 16)
    n = 16 * 64
    K = p.rng.normal(size=(1, 1, n, d)) * 0.3
    V = p.rng.normal(size=K.shape)
    far = np.arange(n) // 64 % 4 == 1
    V[0, 0, far] *= 2.0 ** by
    V[0, 0, far, :d // 2] = 0
    K[..., 0] = 0
    K[0, 0, far, 0] = -64.0
    p.write(K, V, [0])
    Q = p.rng.normal(size=(1, G, t, d))
    Q[..., 0] = 0
    compare(*attend(p, Q, [n], ws=ws), d)
    Q[..., 0] = 64.0                                                          # scores 4096 / sqrt(d) lower there
    O, lse, ref = attend(p, Q, [n], ws=ws)
    compare(O, lse, ref, d)
    assert np.abs(O).max() < 4


@WIDE
@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 24, 2.0 ** 60, 2.0 ** 110])
def test_scores_far_from_zero(wide, size, d, t, G):
    """Whole scores of up to 6 * size, of both signs, a few of them equal: the greatest alone count from 2^24 on."""
    p = Pair(1, 1, d, 64, 6)
    n = 6 * 64
    K = np.zeros((1, 1, n, d))
    K[..., 0] = p.rng.choice(so.LEVELS, size=n)
    V = p.rng.normal(size=K.shape)
    p.write(K, V, [0])
    Q = np.zeros((1, G, t, d))
    Q[..., 0] = size
    for sign in (1, -1):
        compare(*attend(p, Q * sign, [n], scale=1.0), d)


@WIDE
@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("first", [22, 25, 26, 27, 28, 31])
def test_scores_farther_apart_than_weights_reach(wide, first, up, d, t, G):
    """The greatest scores double from block to block, 3 * 2^first and on, up or down the cache: outputs are the mean of the two values whose keys
    are the greatest of all. A weight is rounded to 2^-8 of it, and so is the output."""
    p = Pair(1, 1, d, 64, 5)
    n = 5 * 64
    K = np.zeros((1, 1, n, d))
    best = []
    for j in range(5):
        of = 2.0 ** (j if up else 4 - j)
        K[0, 0, 64 * j:64 * j + 64, 0] = p.rng.choice([0, 0.5, 1.0, 1.5], size=64) * of
        best.append(64 * j + p.rng.permutation(64)[:2])
        K[0, 0, best[-1], 0] = 3.0 * of
    V = p.rng.normal(size=K.shape)
    p.write(K, V, [0])
    Q = np.zeros((1, G, t, d))
    Q[..., 0] = 2.0 ** first
    O, lse, ref = attend(p, Q, [n], scale=1.0)
    compare(O, lse, ref, d)
    two = np.stack([so.stored(f64(bf16(V[0, 0, i])), d) for i in best[4 if up else 0]])
    assert (np.abs(O - two.mean(0)) <= 2.0 ** -7 * np.abs(two).mean(0) + 2.0 ** -100).all()


@WIDE
@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("keys", [1, 2, 3])
def test_log_sum_exps_of_few_keys(wide, keys, d, t, G):
    """Where next to nothing is summed the log-sum-exp is as exact as a score: 2^-21 and the scores' own bound."""
    p = Pair(24, 1, d, 64, 1, seed=keys)
    p.fill([keys] * 24)
    Q = p.rng.normal(size=(24, G, t, d)) * 0.3
    O, lse, ref = attend(p, Q, [keys] * 24)
    compare(O, lse, ref, d)
    if keys == 1 and t * G <= 32:                                              # the one value as it is stored
        for b in range(24):
            assert (O[b] == ref["O"][b]).all()


@WIDE
@pytest.mark.parametrize("d,t,G", KINDS)
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("gap,size", [(60, 99), (100, 9), (120, 40), (124, 9), (124, 99)])
def test_large_values_of_small_weight(wide, gap, size, up, d, t, G):
    """Half of the channels have values of 2^size in one block alone, whose scores are 2^-gap of the other's: before it and behind it."""
    p = Pair(1, 1, d, 64, 2)
    K, V = np.zeros((1, 1, 128, d)), p.rng.normal(size=(1, 1, 128, d))
    low = slice(0, 64) if up else slice(64, 128)
    high = slice(64, 128) if up else slice(0, 64)
    K[0, 0, low, 0] = -1
    V[0, 0, high, :d // 2] = 0
    V[0, 0, low] *= 2.0 ** size
    V[0, 0, low, d // 2:] = 0
    p.write(K, V, [0])
    Q = np.zeros((1, G, t, d))
    Q[..., 0] = gap * np.log(2)                                               # (in bf16: 2^-8 of it more at most)
    O, lse, ref = attend(p, Q, [128], scale=1.0)
    compare(O, lse, ref, d)
    if size - gap > -110:
        some = np.abs(ref["O"]) >= 2.0 ** (size - gap - 8)                      # (codes of 64 equal weights may add up to nothing)
        assert some[..., :d // 2].any() and (O[some] != 0).all()


@WIDE
@pytest.mark.parametrize("d,t,G", KINDS)
def test_small_and_large_keys(wide, d, t, G):
    """Runs of channels 2^-100 .. 2^100 apart, each with a query that brings it back."""
    p = Pair(1, 1, d, 64, 4)
    e = np.repeat(p.rng.integers(-100, 101, size=d // 32), 32)
    K = p.rng.normal(size=(1, 1, 256, d)) * 2.0 ** e
    p.write(K, p.rng.normal(size=K.shape), [0])
    compare(*attend(p, p.rng.normal(size=(1, G, t, d)) * 2.0 ** -e, [256], causal=t < 50), d)


@pytest.mark.parametrize("d,t,G", [(64, 1, 8), (128, 3, 1), (64, 40, 1), (128, 70, 1)])
def test_few_rows_of_a_long_cache(d, t, G):
    table = np.random.default_rng(2).integers(0, 40, size=(1, 400))
    p = Pair(1, 1, d, 64, 400, table=table, pages=40)
    one = Pair(1, 1, d, 64, 40, 3, np.arange(40).reshape(1, 40), 40)
    one.gpu = rb.fourbit_of(p.gpu.k_codes, p.gpu.v_codes, p.gpu.scales, p.gpu.k_mean, one.gpu.table, 64)
    one.fill([2560], spread=0.5)
    p.ref.held = one.ref.held
    Q = video_like(p.rng, 1, G, t, d)
    for n in (25600, 25537):
        compare(*attend(p, Q, [n], causal=True), d)


def test_offsets_past_32_bits():
    """The same tokens in the first and in the last pages of a pool of more than 4 GiB of codes for K alone."""
    pages, hk, d, block = 64000, 8, 128, 128
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 10 GB")
    gpu = rb.allocate_cache(2, hk, d, block, pages, 3, DEV, bits=4)
    assert gpu.k_codes.numel() > 1 << 32 and gpu.v_codes.numel() > 1 << 32
    gpu.table.copy_(torch.tensor([[1, 0, 2], [pages - 1, pages - 3, pages - 2]]))
    rng = np.random.default_rng(0)
    K, V = (bf16(np.repeat(rng.normal(size=(1, hk, 300, d)), 2, axis=0)) for _ in range(2))
    rb.rsa_fourbit_write(gpu, rb.make_rows(K), K, V, i32([0, 0]))
    R, S = torch.zeros_like(K), torch.zeros_like(V)
    rb.rsa_fourbit_read(gpu, rb.make_rows(K), i32([0, 0]), None, R, S)
    assert torch.equal(R[0], R[1]) and torch.equal(S[0], S[1]) and (R - K).abs().max() <= 2.0 ** -2 * K.abs().max()
    for t in (5, 50):
        Q = bf16(np.repeat(rng.normal(size=(1, hk, t, d)), 2, axis=0))
        O = torch.zeros_like(Q)
        rb.rsa_fourbit_attn(gpu, rb.make_rows(Q), Q, i32([300, 300]), None, 0.0, 0, None, None, 0, O)
        assert torch.equal(O[0], O[1]) and O.abs().max() > 0


@pytest.mark.parametrize("d,block,G,t", [(64, 64, 1, 1), (128, 128, 2, 2)])
def test_more_short_sequences_than_compute_units(d, block, G, t):
    """300 tiles of one launch: four waves to each, where fewer tiles have eight."""
    p = Pair(60, 5, d, block, 5, table=np.random.default_rng(1).integers(0, 9, size=(60, 5)), pages=9)
    one = Pair(1, 5, d, block, 9, 3, np.arange(9).reshape(1, 9), 9)
    one.gpu = rb.fourbit_of(p.gpu.k_codes, p.gpu.v_codes, p.gpu.scales, p.gpu.k_mean, one.gpu.table, block)
    one.fill([9 * block], spread=0.5)
    p.ref.held = one.ref.held
    lens = [int(n) for n in p.rng.integers(0, 5 * block + 1, size=60)]
    Q = video_like(p.rng, 60, 5 * G, t, d)
    compare(*attend(p, Q, lens, [min(t, n) for n in lens], causal=True), d)


def test_rows_past_32_bits():
    """Heads 2^32 elements apart: what is written, read, attended and turned there is what it is in a small tensor."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 100 GB")
    t, d, far = 70, 64, (1 << 32) + 64
    rng = np.random.default_rng(0)
    big = [torch.empty(far + t * d, dtype=torch.bfloat16, device=DEV).as_strided((1, 2, t, d), (8, far, d, 1)) for _ in range(5)]
    small = [bf16(rng.normal(size=(1, 2, t, d))) for _ in range(3)]
    for x, y in zip(big, small):
        x.copy_(y)
    outs = []
    for K, V, Q, R, S in ((*big,), (*small, torch.zeros_like(small[0]), torch.zeros_like(small[0]))):
        p = Pair(1, 2, d, 64, 2)
        rows = rb.make_rows(K)
        rb.rsa_fourbit_write(p.gpu, rows, K, V, i32([0]))
        rb.rsa_fourbit_read(p.gpu, rows, i32([0]), None, R, S)
        kept = R.clone(memory_format=torch.contiguous_format), S.clone(memory_format=torch.contiguous_format)
        rb.rsa_fourbit_attn(p.gpu, rows, Q, i32([t]), None, 0.0, rb.RSA_CACHE_CAUSAL, None, None, 0, R)
        rot = rb.make_rotary(torch.full((32,), 0.1, dtype=torch.float64, device=DEV))
        rb.rsa_rotary_apply(rot, rows, Q, S)
        outs.append([*kept, R.clone(memory_format=torch.contiguous_format), S.clone(memory_format=torch.contiguous_format)])
    for x, y in zip(*outs):
        assert torch.equal(x, y) and x.abs().max() > 0


def test_prompts_of_many_tiles():
    """More workgroups than the chip takes at once, the last tokens first: against rows taken one at a time by the other kernel."""
    p = Pair(1, 8, 64, 64, 64)
    n = 4096
    K = bf16(video_like(p.rng, 1, 8, n, 64))
    rb.rsa_fourbit_write(p.gpu, rb.make_rows(K), K, K, i32([0]))
    Q = bf16(video_like(p.rng, 1, 16, n, 64))
    O = torch.zeros_like(Q)
    rows = rb.make_rows(Q)
    rb.rsa_fourbit_attn(p.gpu, rows, Q, i32([n]), None, 0.0, rb.RSA_CACHE_CAUSAL, None, None, 0, O)
    for i in (0, 1, 63, 64, 1000, 2047, 4095):
        q = Q[:, :, i:i + 1].contiguous()
        o = torch.zeros_like(q)
        rb.rsa_fourbit_attn(p.gpu, rb.make_rows(q), q, i32([i + 1]), None, 0.0, 0, None, None, 0, o)
        # each is within 2^-7 (rounding of weights and output) of the same number, of values of at most 4 on average
        assert (o[:, :, 0].float() - O[:, :, i].float()).abs().max() <= 2.0 ** -6 * o.float().abs().max().clamp(min=1)


def test_the_same_call_twice_gives_the_same_bits():
    p = Pair(2, 2, 128, 64, 40)
    p.fill([2500, 1300])
    for t in (1, 40):
        Q = bf16(p.rng.normal(size=(2, 4, t, 128)))
        rows = rb.make_rows(Q)
        ws = torch.empty(max(256, rb.rsa_fourbit_workspace_bytes(p.gpu, rows)), dtype=torch.uint8, device=DEV)
        outs = []
        for _ in range(3):
            O = torch.zeros_like(Q)
            rb.rsa_fourbit_attn(p.gpu, rows, Q, i32([2500, 1300]), None, 0.0, 0, None, None, 0, O, None, ws)
            ws.random_()
            outs.append(O)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ---- pages ---------------------------------------------------------------------------------------
def run_assign(table, free, free_count, kv_len, add, t, block, pages, shared=None, in_place=False, maps=True):
    batch = len(kv_len)
    dev = dict(dtype=torch.int32, device=DEV)
    T = torch.tensor(np.asarray(table), **dev).contiguous()
    F = torch.full((pages,), -77, **dev)
    F[:len(free)] = torch.tensor(free, **dev) if len(free) else F[:0]
    kv, fc = i32(kv_len), i32([free_count])
    kv_new, left = (kv, fc) if in_place else (torch.full((batch,), -9, **dev), torch.full((1,), -9, **dev))
    start, count = torch.full((batch,), -9, **dev), torch.full((batch,), -9, **dev)
    pos = torch.full((batch, t), -9, **dev) if maps else None
    slot = torch.full((batch, t), -9, dtype=torch.int64, device=DEV) if maps else None
    rb.rsa_cache_assign(rb.pages_of(T, F, block), t, kv, i32(add), fc, kv_new, left, start, count, pos, slot, i32(shared))
    want = so.assign(table, free, free_count, kv_len, add, t, block, pages, shared)
    assert T.tolist() == want[0].tolist()
    assert int(left) == len(want[1]) and F[:int(left)].tolist() == want[1]
    assert kv_new.tolist() == want[2] and start.tolist() == want[3] and count.tolist() == want[4]
    if maps:
        assert pos.tolist() == want[5].tolist() and slot.tolist() == want[6].tolist()
    return want


def some_state(rng, batch, width, block, spare, holes=False):
    kv = [int(rng.integers(0, width * block + 1)) for _ in range(batch)]
    n = sum(-(-x // block) for x in kv)
    pages = n + spare + 5
    order = rng.permutation(pages).tolist()
    table = np.full((batch, width), -1)
    for b, x in enumerate(kv):
        for e in range(-(-x // block)):
            table[b, e] = order.pop()
            if holes and rng.random() < 0.2:
                table[b, e] = rng.choice([-1, -5, pages, 2 ** 31 - 1])
    return kv, table, order[:spare], pages


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,width,block,t,spare", [(1, 4, 64, 1, 0), (5, 7, 64, 3, 2), (32, 40, 64, 1, 50), (48, 30, 128, 700, 400), (70, 9, 64, 130, 60),
                                                       (1500, 6, 64, 2, 300), (2500, 3, 16, 40, 900), (3, 500, 1, 450, 700), (2, 20000, 64, 5000, 300)])
def test_assign(batch, width, block, t, spare, in_place):
    for seed in range(3):
        rng = np.random.default_rng([seed, batch])
        kv, table, free, pages = some_state(rng, batch, width, block, spare, holes=seed == 2)
        add = rng.integers(-width * block if seed else 0, t + 2, size=batch)
        if seed == 1:
            add = np.where(rng.random(batch) < 0.6, rng.integers(0, t + 1, size=batch), add)     # few go
        shared = rng.integers(-1, width + 1, size=batch).tolist() if seed == 2 else None
        run_assign(table, free, len(free), kv, add.tolist(), t, block, pages, shared, in_place, maps=seed != 1)


@pytest.mark.parametrize("batch", [1, 2, 3, 7, 9, 16, 17])
@pytest.mark.parametrize("t", [300, 4097, 9000])
def test_assign_long_prompts(batch, t):
    """Hundreds and thousands of pages to a sequence, shared out over waves; the last sequence finds the list short."""
    rng = np.random.default_rng(batch)
    held = rng.integers(0, 50, size=batch)
    need = [-(-(int(x) + t) // 3) - -(-int(x) // 3) for x in held]
    pages = sum(need) + sum(-(-int(x) // 3) for x in held) + 3
    order = rng.permutation(pages).tolist()
    table = np.full((batch, 3100), -1)
    for b, x in enumerate(held):
        for e in range(-(-int(x) // 3)):
            table[b, e] = order.pop()
    for spare in (sum(need), sum(need) - 1):
        run_assign(table, order[:spare], spare, held.tolist(), [t] * batch, t, 3, pages, maps=t * batch < 40000)


def test_assign_at_its_edges():
    # no page is left; the one that needs none is served
    run_assign([[3, -1], [4, -1]], [], 0, [64, 10], [1, 1], 1, 64, 8)
    # the first asks for more than there is: those behind it that need a page get none either
    run_assign([[-1] * 4, [-1] * 4, [5, -1, -1, -1]], [1, 2], 2, [0, 0, 3], [200, 1, 1], 200, 64, 8)
    # a table that is full asks for none: the next is served; a free_count beyond the list, and below zero
    run_assign([[0, 1], [2, -1]], [7, 6], 2, [128, 64], [1, 1], 4, 64, 8)
    run_assign([[-1, -1]], list(range(8)), 99, [0], [100], 100, 64, 8)
    run_assign([[-1, -1]], list(range(8)), -3, [0], [100], 100, 64, 8)
    # lengths outside the table, more new tokens than rows, more taken than there are
    run_assign([[0, 1], [2, 3], [4, 5]], [6], 1, [1000, -5, 70], [1, 3, -1000], 2, 64, 8)
    # a list that is full takes no more
    run_assign([[0, 1]], list(range(4)), 4, [128], [-128], 1, 64, 4)
    # what is given back is taken in the same call
    run_assign([[0, 1], [-1, -1]], [], 0, [128, 0], [-128, 128], 128, 64, 4)
    # a shared prefix stays out of the list
    run_assign([[0, 1, 2], [0, 1, 3]], [], 0, [192, 192], [-192, -192], 1, 64, 4, shared=[2, 3])


# ---- rotary positions ----------------------------------------------------------------------------
def run_rotary(rng, b, hq, hk, t, d, pairs, pairing, layout="bhtd", axis_pairs=None, factor=1.0, inverse=False, start=None, count=None, positions=None,
               in_place=False, freq=None, x=None):
    axis_pairs = axis_pairs or [pairs]
    freq = 10000.0 ** (-np.arange(pairs) / pairs) if freq is None else freq
    rot = rb.make_rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), pairing, axis_pairs, factor)
    Q, K = (bf16(rng.normal(size=(b, h, t, d)) if x is None else x[:, :h], layout) for h in (hq, max(hk, 1)))
    want = []
    pos = np.asarray(positions) if positions is not None else np.asarray(start if start is not None else [0] * b)[None, :, None] + np.arange(t)
    n = np.full(b, t) if count is None else np.asarray(count)
    for X in (Q, K):
        want.append((f64(X), *so.rotate(f64(X), pos, freq, pairing, axis_pairs, factor, inverse)))
    Qr, Kr = (Q, K) if in_place else (torch.full_like(Q, 7.0), torch.full_like(K, 7.0))
    p = None if positions is None else torch.tensor(np.asarray(positions), dtype=torch.int32, device=DEV).contiguous()
    flags = rb.RSA_ROTARY_INVERSE if inverse else 0
    if hk:
        rb.rsa_rotary_apply(rot, rb.make_rows(Q), Q, Qr, rb.make_rows(K), K, Kr, p, i32(start), i32(count), flags)
    else:
        rb.rsa_rotary_apply(rot, rb.make_rows(Q), Q, Qr, positions=p, start=i32(start), count=i32(count), flags=flags)
    for got, (before, y, size) in list(zip((f64(Qr), f64(Kr)), want))[:2 if hk else 1]:
        for i in range(b):
            m = max(0, min(t, n[i]))
            assert np.array_equal(got[i, :, m:], before[i, :, m:] if in_place else np.full_like(got[i, :, m:], 7.0))
            g, w, s = got[i, :, :m], y[i, :, :m], size[i, :, :m]
            bound = 2.0 ** -8 * np.abs(w) + 2.0 ** -21 * s
            bound[..., 2 * pairs:] = 0
            ok = np.isfinite(w)
            assert np.array_equal(ok, np.isfinite(g))
            off = np.abs(g[ok] - w[ok])
            assert (off <= bound[ok]).all(), (off / np.maximum(bound[ok], 1e-30)).max()
    return f64(Qr), f64(Kr)


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("d,pairs", [(128, 64), (128, 32), (64, 32), (64, 16), (128, 55), (64, 1), (128, 63), (64, 29), (8, 4), (8, 3), (24, 12), (40, 8), (72, 36), (1024, 512), (200, 17)])
def test_rotary(d, pairs, pairing):
    rng = np.random.default_rng([d, pairs])
    run_rotary(rng, 2, 3, 2, 5, d, pairs, pairing, start=[0, 70000])
    run_rotary(rng, 3, 1, 4, 7, d, pairs, pairing, "bthd", start=[5, 9, 100], count=[7, 0, 3], in_place=True, inverse=True, factor=1.2)
    if pairs > 3:
        axes = [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]
        pos = rng.integers(-3000, 3000, size=(3, 2, 6))
        run_rotary(rng, 2, 2, 0, 6, d, pairs, pairing, axis_pairs=axes, positions=pos)
        run_rotary(rng, 2, 2, 1, 6, d, pairs, pairing, axis_pairs=[0, pairs], positions=pos[:2], count=[6, 1])


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 24 + 1, 2 ** 31 - 40, -2 ** 31])
def test_rotary_far_positions(far):
    """Angles of 2^31 radians: fp64 leaves 2^-22 of one in the oracle as in the kernel (a step of 2^-22 at 2^31), a fifth of the bound."""
    rng = np.random.default_rng(1)
    run_rotary(rng, 1, 2, 2, 33, 128, 64, "half", start=[far])
    run_rotary(rng, 1, 2, 2, 33, 64, 32, "interleaved", positions=far + np.arange(33).reshape(1, 1, 33))


def test_rotary_leaves_what_does_not_turn():
    """Infinities and NaN in the channels behind the pairs are copied and reach no other."""
    x = np.random.default_rng(0).normal(size=(1, 2, 3, 64))
    x[..., 20], x[..., 21], x[..., 63] = np.inf, -np.inf, np.nan
    for pairing in ("half", "interleaved"):
        for in_place in (False, True):
            q, k = run_rotary(np.random.default_rng(0), 1, 2, 2, 3, 64, 10, pairing, x=x, in_place=in_place)
            assert np.isfinite(q[..., :20]).all() and np.isposinf(q[..., 20]).all() and np.isneginf(q[..., 21]).all() and np.isnan(q[..., 63]).all()


def test_rotary_gradient():
    """The inverse is the transpose: <turn(x), g> = <x, turn back(g)>, and differences of the turned rows along g agree with it."""
    rng = np.random.default_rng(2)
    for pairing in ("half", "interleaved"):
        x, g = rng.normal(size=(2, 1, 2, 9, 64))
        y, _ = run_rotary(rng, 1, 2, 2, 9, 64, 24, pairing, x=x, start=[1000], factor=1.3)
        back, _ = run_rotary(rng, 1, 2, 2, 9, 64, 24, pairing, x=g, start=[1000], factor=1.3, inverse=True)
        xb, gb = f64(bf16(x)), f64(bf16(g))
        y2, _ = run_rotary(rng, 1, 2, 2, 9, 64, 24, pairing, x=f64(bf16(xb + gb)), start=[1000], factor=1.3)
        # every output and input is off by at most half a step, 2^-8: of the products' magnitudes, twice
        left, right, size = (y * gb).sum(), (xb * back).sum(), (np.abs(y * gb) + np.abs(xb * back)).sum()
        assert abs(left - right) <= 2.0 ** -8 * size
        step = ((y2 - y) * gb).sum()
        assert abs(step - (gb * back).sum()) <= 2.0 ** -8 * (np.abs(y2 * gb) + np.abs(y * gb) + np.abs(gb * back) + np.abs(y2 * gb)).sum() * 1.5


def test_rotary_of_many_tokens():
    """More rows than a round of workgroups, so that a thread walks several heads, of two tensors with strides of their own."""
    rng = np.random.default_rng(4)
    run_rotary(rng, 1, 5, 3, 20000, 128, 64, "half", "bthd", start=[77])
    run_rotary(rng, 2, 3, 2, 12000, 64, 32, "interleaved", start=[77, 0], count=[11999, 6000])


# ---- together ------------------------------------------------------------------------------------
def serve(bits, captured):
    """Requests that arrive, grow token by token, go and make room: every step against the oracle's pages and attention."""
    B, hq, hk, d, block, width, pages, t = 4, 4, 2, 64, 64, 6, 14, 70
    rng = np.random.default_rng(7)
    freq, factor = rb.rsa_rotary_frequencies(24, 10000.0, rb.RSA_ROTARY_PARTS, 4.0, 256.0)
    rot = rb.make_rotary(torch.tensor(freq, dtype=torch.float64, device=DEV), "half", None, factor)
    cache = rb.allocate_cache(B, hk, d, block, pages, width, DEV, bits=bits)
    Cache = so.Cache if bits == 4 else co.Cache
    free = list(rng.permutation(pages))
    dev = dict(dtype=torch.int32, device=DEV)
    F = torch.tensor(free, **dev)
    rec = rb.pages_of(cache.table, F, block)
    kv, fc, start, count, add = torch.zeros(B, **dev), torch.tensor([pages], **dev), torch.zeros(B, **dev), torch.zeros(B, **dev), torch.zeros(B, **dev)
    Q, K, V = (torch.zeros(B, h, t, d, dtype=torch.bfloat16, device=DEV) for h in (hq, hk, hk))
    O = torch.zeros_like(Q)
    lse = torch.zeros(B, hq, t, device=DEV)
    pos, slot = torch.zeros(B, t, **dev), torch.zeros(B, t, dtype=torch.int64, device=DEV)
    size = rb.rsa_fourbit_workspace_bytes(cache, rb.make_rows(Q)) if bits == 4 else rb.rsa_cache_workspace_bytes(cache, rb.make_rows(Q))[1]
    ws = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
    step = lambda: rb.serve_step(cache, rec, rot, Q, K, V, O, kv, add, fc, start, count, pos, slot, None, lse, ws)
    graph = None
    table, held, nfree = np.full((B, width), -1), [0] * B, free
    ref = Cache(hk, d, block, table, pages)
    refused = 0
    for i, adds in enumerate([[70, 3, 64, 0], [1, 1, 1, 70], [70, 1, 1, 1], [70, 70, 70, 1], [1, 70, 70, 70], [70, 70, 1, 70], [-500, 1, 1, 70], [5, -40, 1, 1],
                              [70, 70, 70, 70], [1, 1, 1, 1]]):
        x = [bf16(rng.normal(size=(B, h, t, d))) for h in (hq, hk, hk)]
        for dst, src in zip((Q, K, V), x):
            dst.copy_(src)
        add.copy_(torch.tensor(adds))
        O.fill_(7.0)
        lse.fill_(7.0)
        if captured and i == 1:                                   # (the first step has run eagerly)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        table, nfree, new, st, ct, p, s = so.assign(table, nfree, len(nfree), held, adds, t, block, pages)
        refused += sum(a > 0 and c == 0 for a, c in zip(adds, ct))
        assert cache.table.tolist() == table.tolist() and kv.tolist() == new and count.tolist() == ct and start.tolist() == st
        assert int(fc) == len(nfree) and F[:len(nfree)].tolist() == [int(z) for z in nfree] and pos.tolist() == p.tolist() and slot.tolist() == s.tolist()
        held = new
        at = np.asarray(st)[None, :, None] + np.arange(t)
        for got, src in ((Q, x[0]), (K, x[1])):
            y, size = so.rotate(f64(src), at, np.array(freq), "half", [24], factor)
            for b in range(B):
                assert (np.abs(f64(got)[b, :, :ct[b]] - y[b, :, :ct[b]]) <= 2.0 ** -8 * np.abs(y[b, :, :ct[b]]) + 2.0 ** -21 * size[b, :, :ct[b]]).all()
                assert torch.equal(got[b, :, ct[b]:], src[b, :, ct[b]:])
        ref.table = table
        ref.write(f64(K), f64(V), st, ct)
        out = ref.attend(f64(Q), held, ct, 0.0, True)
        if bits == 4:
            compare(f64(O), lse.cpu().double().numpy(), out, d)
        else:
            err = np.abs(f64(O) - out["O"])[out["isq"]]
            assert (err <= 2.0 ** -8 * np.abs(out["O"])[out["isq"]] + 2.0 ** -10 * out["A"][out["isq"]]).all()
    assert refused >= 2


@pytest.mark.parametrize("bits", [4, 8])
def test_a_batch_of_requests(bits):
    serve(bits, False)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_batch_of_requests_replayed(bits):
    """One captured step serves all of it: lengths, tables and positions move on inside the graph, with eager work between the replays."""
    serve(bits, True)


def test_selected_blocks_of_the_four_bit_cache():
    """cached_sparse_attention on a cache of 4 bits, on a stream of its own."""
    p = Pair(2, 2, 128, 64, 20)
    p.fill([1100, 700])
    K, V = p.rng.normal(size=(2, 2, 2, 40, 128))
    Q = bf16(p.rng.normal(size=(2, 4, 40, 128)))
    Kd, Vd, O = bf16(K), bf16(V), torch.full_like(Q, 7.0)
    lens, q_len = [1140, 730], [40, 30]
    idx, kept = torch.zeros(2, 2, 3, 8, dtype=torch.int32, device=DEV), torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    kv, ql = i32(lens), i32(q_len)
    lse = torch.full((2, 4, 40), 7.0, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rb.cached_sparse_attention(p.gpu, Kd, Vd, Q, O, kv, ql, 16, 6, idx, kept, lse=lse, stream=side)
    side.synchronize()
    p.ref.write(f64(Kd), f64(Vd), [1100, 700], q_len)
    lists = p.ref.select(f64(Q), lens, q_len, 16, 6, 1, 1, True)
    for (b, h, g), x in lists.items():
        assert int(kept[b, h, g]) == len(x) and idx[b, h, g, :len(x)].tolist() == x
    compare(f64(O), lse.cpu().double().numpy(), p.ref.attend(f64(Q), lens, q_len, 0.0, True, lists, 16), 128)


def test_binding_refusals():
    four, eight = (rb.allocate_cache(2, 2, 64, 64, 4, 2, DEV, bits=n) for n in (4, 8))
    x = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device=DEV)
    rows, z = rb.make_rows(x), i32([0, 0])
    for cache, write, read, attn in ((eight, rb.rsa_fourbit_write, rb.rsa_fourbit_read, rb.rsa_fourbit_attn), (four, rb.rsa_cache_write, rb.rsa_cache_read, rb.rsa_cache_attn)):
        with pytest.raises(ValueError, match="bits"):
            write(cache, rows, x, x, z)
        with pytest.raises(ValueError, match="bits"):
            read(cache, rows, z, None, x, x.clone())
        with pytest.raises(ValueError, match="bits"):
            attn(cache, rows, x, z, None, 0.0, 0, None, None, 0, x)
    with pytest.raises(ValueError):
        rb.allocate_cache(1, 1, 64, 64, 1, 1, DEV, bits=2)
    with pytest.raises(ValueError):
        rb.rsa_fourbit_write(four, rows, x, x[:, :, :2], z)
    rot = rb.make_rotary(torch.ones(32, dtype=torch.float64, device=DEV))
    for bad in (dict(Q=x.float()), dict(Qr=x[:, :1]), dict(start=z.long()), dict(count=i32([1])), dict(positions=torch.zeros(2, 4, dtype=torch.int32, device=DEV))):
        args = dict(rotary=rot, rows_q=rows, Q=x, Qr=x)
        with pytest.raises(ValueError):
            rb.rsa_rotary_apply(**{**args, **bad})
    rec = rb.pages_of(torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), 64)
    one = i32([1])
    with pytest.raises(ValueError):
        rb.rsa_cache_assign(rec, 1, z, z, z, z.clone(), one, z.clone(), z.clone())
    with pytest.raises(rb.RsaError):
        rb.rsa_cache_assign(rec, 1, z, z.clone(), one, z, one, z, z.clone())        # start over the lengths
    with pytest.raises(ValueError, match="table"):
        rb.serve_step(four, rec, rot, x, x, x, x, z, z, one, z, z)
    # nothing of a step that is refused has happened
    rec = rb.pages_of(four.table, torch.arange(4, dtype=torch.int32, device=DEV), 64)
    half = rb.make_rotary(torch.ones(32, dtype=torch.float64, device=DEV))
    good = dict(cache=four, pages=rec, rotary=half, Q=x, K=x.clone(), V=x.clone(), O=x.clone(), kv_len=i32([0, 0]), add=i32([3, 3]), free_count=i32([4]), start=i32([0, 0]),
                count=i32([0, 0]))
    wide = torch.zeros(2, 2, 3, 128, dtype=torch.bfloat16, device=DEV)
    odd = torch.zeros(2, 2, 3, 68, dtype=torch.bfloat16, device=DEV)[..., :64]          # rows 136 bytes apart
    for bad in (dict(K=x[:, :, :2].contiguous(), V=x[:, :, :2].contiguous()), dict(O=x[:, :, :2]), dict(V=x[:, :1]), dict(Q=wide, O=wide), dict(K=x[:, :1].contiguous(), V=x[:, :1].contiguous()),
                dict(lse=torch.zeros(2, 2, 2, device=DEV)), dict(rotary=rb.make_rotary(torch.ones(33, dtype=torch.float64, device=DEV))),
                dict(rotary=rb.make_rotary(torch.ones(32, dtype=torch.float64, device=DEV), axis_pairs=[16, 16])),
                dict(pages=rb.pages_of(four.table, torch.arange(4, dtype=torch.int32, device=DEV), 128)),
                dict(pages=rb.pages_of(four.table, torch.arange(5, dtype=torch.int32, device=DEV), 64)), dict(K=x), dict(ws=torch.zeros(1, device=DEV).expand(2)),
                dict(ws=torch.zeros(4096, dtype=torch.uint8, device=DEV)[16:]), dict(V=torch.zeros(2 * 2 * 3 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(2, 2, 3, 64)),
                dict(Q=odd, O=odd), dict(K=odd, V=odd)):
        with pytest.raises((ValueError, RuntimeError)):
            rb.serve_step(**{**good, **bad})
    assert int(good["free_count"]) == 4 and good["kv_len"].tolist() == [0, 0] and (four.table == -1).all()
    rb.serve_step(**good)
    assert int(good["free_count"]) == 2 and good["kv_len"].tolist() == [3, 3]


def step_of(batch, hq, hk, d, t, width=1, pages=4, strides=None):
    """Arguments of a step that would be served: zeros, `t` new tokens for each sequence."""
    def rows(h):
        if strides is None:
            return torch.zeros(batch, h, t, d, dtype=torch.bfloat16, device=DEV)
        n = 1 + sum((m - 1) * s for m, s in zip((batch, h, t, d), strides))
        return torch.zeros(n, dtype=torch.bfloat16, device=DEV).as_strided((batch, h, t, d), strides)
    cache = rb.allocate_cache(batch, hk, d, 64, pages, width, DEV, bits=4)
    n = lambda x: torch.full((batch,), x, dtype=torch.int32, device=DEV)
    return dict(cache=cache, pages=rb.pages_of(cache.table, torch.arange(pages, dtype=torch.int32, device=DEV), 64),
                rotary=rb.make_rotary(torch.ones(d // 2, dtype=torch.float64, device=DEV)), Q=rows(hq), K=rows(hk), V=rows(hk), O=rows(hq), kv_len=n(0), add=n(t),
                free_count=i32([pages]), start=n(-9), count=n(-9))


def refused(step, **bad):
    """The step raises, and lengths, table and list are what they were."""
    with pytest.raises((ValueError, RuntimeError)):
        rb.serve_step(**{**step, **bad})
    torch.cuda.synchronize()
    assert int(step["free_count"]) == step["pages"].desc.pages and (step["kv_len"] == 0).all() and (step["cache"].table == -1).all() and (step["count"] == -9).all()


def test_a_step_whose_values_are_its_keys_or_queries_is_refused():
    """Queries and keys are turned where they stand, before the values are written."""
    step = step_of(2, 2, 2, 64, 3)
    refused(step, V=step["K"])
    refused(step, V=step["Q"])
    fused = torch.zeros(2, 3, 6, 64, dtype=torch.bfloat16, device=DEV).permute(0, 2, 1, 3)        # one product's rows: queries, keys, values of a token
    Q, K, V = fused[:, :2], fused[:, 2:4], fused[:, 4:]
    Q.copy_(bf16(np.random.default_rng(0).normal(size=(2, 2, 3, 64))))
    K.copy_(Q)
    V.copy_(Q)
    rb.serve_step(**{**step, "Q": Q, "K": K, "V": V, "O": Q})
    assert step["kv_len"].tolist() == [3, 3]
    R, S = torch.zeros_like(step["K"]), torch.zeros_like(step["V"])
    rb.rsa_fourbit_read(step["cache"], rb.make_rows(R), i32([0, 0]), None, R, S)
    want = np.stack([so.stored(x, 64) for x in f64(V).reshape(-1, 64)]).reshape(2, 2, 3, 64)
    np.testing.assert_array_equal(f64(S), want)                                  # as they came


@pytest.mark.parametrize("sizes", [dict(batch=29128, hq=1, hk=1, d=128, t=1024, strides=(8, 8, 128, 1)),       # 29128 * 1024 * 18 / 64 >= 2^23 workgroups of the turning
                                   dict(batch=1, hq=65535, hk=1, d=64, t=1)])                                  # 65536 heads of queries and keys
def test_a_step_too_large_to_be_turned_is_refused(sizes):
    """Sizes that pages and cache take, and rsa_rotary_apply does not: refused before the pages are given out."""
    refused(step_of(**sizes))


class Requests:
    """Pages, lengths and shared prefixes on the GPU and in the oracle, moved on in place step by step."""

    def __init__(self, table, free, kv, shared, block, pages, t):
        dev = dict(dtype=torch.int32, device=DEV)
        self.block, self.pages, self.t, self.batch = block, pages, t, len(kv)
        self.table, self.free, self.kv, self.shared = np.array(table), list(free), list(kv), list(shared)
        self.T, self.F = torch.tensor(np.asarray(table), **dev), torch.tensor(list(free) + [-77] * (pages - len(free)), **dev)
        self.gkv, self.gsh, self.fc = i32(kv), i32(shared), i32([len(free)])
        self.start, self.count = torch.zeros(self.batch, **dev), torch.zeros(self.batch, **dev)

    def step(self, add):
        rb.rsa_cache_assign(rb.pages_of(self.T, self.F, self.block), self.t, self.gkv, i32(add), self.fc, self.gkv, self.fc, self.start, self.count, shared=self.gsh)
        self.table, self.free, self.kv, start, count, _, _ = so.assign(self.table, self.free, len(self.free), self.kv, add, self.t, self.block, self.pages, self.shared)
        assert self.T.tolist() == self.table.tolist() and self.F[:int(self.fc)].tolist() == self.free and self.gkv.tolist() == self.kv
        assert self.start.tolist() == start and self.count.tolist() == count and self.gsh.tolist() == self.shared
        return count


def test_pages_below_a_shared_prefix_come_back():
    """Two sequences on a prefix of two pages; the second goes back to the first page, on, and back again."""
    r = Requests([[0, 1, -1], [0, 1, 2]], [3, 4], [128, 192], [2, 2], 64, 5, 128)
    r.step([0, -128])
    assert sorted(r.free) == [2, 3, 4]
    r.step([0, 128])
    assert r.shared == [2, 1] and len(r.free) == 1
    r.step([0, -128])
    assert sorted(r.free) == [2, 3, 4] and r.table[0].tolist() == [0, 1, -1]


@pytest.mark.parametrize("batch,t", [(3, 1), (5, 40), (200, 7), (1500, 3)])
def test_no_page_is_lost_or_held_twice(batch, t):
    """Sequences on two prefixes grow, are cut anywhere and grow again: every page is on the list, one sequence's or a prefix's."""
    rng = np.random.default_rng(batch)
    block, width, held = 4, 6, 3
    pages = 2 * held + batch * 3
    table, shared, kv = np.full((batch, width), -1), [], []
    for b in range(batch):
        n = int(rng.integers(0, held + 1))
        table[b, :n] = np.arange(n) + b % 2 * held
        shared.append(n)
        kv.append(n * block)
    r = Requests(table, rng.permutation(np.arange(2 * held, pages)).tolist(), kv, shared, block, pages, t)
    for i in range(25):
        r.step(np.where(rng.random(batch) < 0.3, -rng.integers(0, width * block, size=batch), rng.integers(0, t + 1, size=batch)).tolist())
        own = [int(p) for b in range(batch) for e, p in enumerate(r.table[b]) if p >= 0 and e >= r.shared[b]]
        assert sorted(own + r.free) == list(range(2 * held, pages))


def test_no_token_goes_into_a_shared_page():
    """Sequences that end inside a block of their prefix are not served and ask for no page; those behind them in the batch are."""
    cases = [(70, 2), (64, 2), (128, 2), (130, 2), (70, 1), (1, 1), (0, 2), (70, -1), (100, 2)]
    n = [-(-kv // 64) for kv, _ in cases]
    table = [[10 * b + e if e < n[b] else -1 for e in range(4)] for b in range(len(cases))]
    for t, add in ((1, 1), (80, 80), (80, 0), (80, -3)):
        r = Requests(table, range(100, 120), [kv for kv, _ in cases], [s for _, s in cases], 64, 200, t)
        count = r.step([add] * len(cases))
        assert [c > 0 for c in count] == [add > 0 and b not in (0, 5, 8) for b in range(len(cases))]


@pytest.mark.parametrize("bits", [4, 8])
def test_a_shared_prefix_stays_what_it_is(bits):
    """Two sequences on a prefix of two pages, in a captured step: one is cut into its second page, asks for more, goes back to the border, grows."""
    rng = np.random.default_rng(3)
    cache = rb.allocate_cache(2, 1, 64, 64, 8, 4, DEV, bits=bits)
    cache.table.copy_(torch.tensor([[0, 1, -1, -1], [0, 1, -1, -1]]))
    rec = rb.pages_of(cache.table, torch.tensor([2, 3, 4, 5, 6, 7, 0, 0], dtype=torch.int32, device=DEV), 64)
    K, V = (bf16(rng.normal(size=(2, 1, 128, 64))) for _ in range(2))
    (rb.rsa_fourbit_write if bits == 4 else rb.rsa_cache_write)(cache, rb.make_rows(K), K, V, i32([0, 0]), i32([128, 0]))
    before = [x[:2].clone() for x in (cache.k_codes, cache.v_codes, cache.scales, cache.k_mean)]
    rot = rb.make_rotary(torch.ones(32, dtype=torch.float64, device=DEV))
    kv, add, fc, shared, start, count = i32([128, 128]), i32([0, 0]), i32([6]), i32([2, 2]), i32([0, 0]), i32([0, 0])
    Q, K, V, O = (bf16(rng.normal(size=(2, 1, 40, 64))) for _ in range(4))
    step = lambda: rb.serve_step(cache, rec, rot, Q, K, V, O, kv, add, fc, start, count, shared=shared)
    step()                                                        # (eagerly, of no token)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    # (adds, lengths, shared entries, pages left); the first sequence grows on its own pages beside it
    for adds, lens, own, left in (([10, -50], [138, 78], [2, 2], 5), ([10, 40], [148, 78], [2, 2], 5), ([10, -14], [158, 64], [2, 2], 5), ([10, 40], [168, 104], [2, 1], 4),
                                  ([10, 40], [178, 144], [2, 1], 3), ([-100, -144], [78, 0], [2, 1], 6), ([1, 40], [78, 40], [2, 0], 5)):
        add.copy_(torch.tensor(adds))
        graph.replay()
        torch.cuda.synchronize()
        assert (kv.tolist(), shared.tolist(), int(fc)) == (lens, own, left)
        for x, y in zip((cache.k_codes, cache.v_codes, cache.scales, cache.k_mean), before):
            assert torch.equal(x[:2], y)


@pytest.mark.parametrize("far", [2 ** 31 - 40, -2 ** 31, 12345678])
def test_rotary_many_radians_a_position(far):
    """Frequencies of up to 1000 radians a position, so that angles reach 2^41, where a step of 64 bits is 2^-11 radians: what they round away counts."""
    freq = 1000.0 ** (1 - np.arange(64) / 32)
    run_rotary(np.random.default_rng(5), 1, 2, 2, 33, 128, 64, "half", start=[far], freq=freq)
    run_rotary(np.random.default_rng(6), 1, 2, 2, 33, 64, 32, "interleaved", positions=far + np.arange(33).reshape(1, 1, 33), freq=freq[:32])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d,block", [(64, 64), (128, 128)])
def test_means_after_a_cut_are_renewed_by_the_next_write(bits, d, block):
    """A sequence is cut inside a block whose last tokens made its mean, grows by one token, and the selection ranks the block by what it holds now."""
    rng = np.random.default_rng(bits)
    width, hk = 6, 2
    cache = rb.allocate_cache(2, hk, d, block, 12, width, DEV, bits=bits)
    ref = (so.Cache if bits == 4 else co.Cache)(hk, d, block, np.full((2, width), -1), 12)
    write = rb.rsa_fourbit_write if bits == 4 else rb.rsa_cache_write
    t = 5 * block
    rec = rb.pages_of(cache.table, torch.arange(12, dtype=torch.int32, device=DEV), block)
    kv, fc, start, count = i32([0, 0]), i32([12]), i32([0, 0]), i32([0, 0])
    table, free, held = np.full((2, width), -1), list(range(12)), [0, 0]
    kept_blocks = []
    for add in ([t, t - 3], [-block - 20, -block // 2], [1, 2], [1, 1]):
        rb.rsa_cache_assign(rec, t, kv, i32(add), fc, kv, fc, start, count)
        table, free, held, st, ct, _, _ = so.assign(table, free, len(free), held, add, t, block, 12)
        assert kv.tolist() == held and cache.table.tolist() == table.tolist()
        K, V = (rng.normal(size=(2, hk, t, d)) for _ in range(2))
        for b in range(2):                                                    # the tokens that the cut takes point one way, and outweigh the block's others
            K[b, :, max(0, held[b] - block - 20):, 0] += 60 if sum(ct) > 4 else 0
        Kd, Vd = bf16(K), bf16(V)
        write(cache, rb.make_rows(Kd), Kd, Vd, start, count)
        ref.table = table
        ref.write(f64(Kd), f64(Vd), st, ct)
        if max(ct) == 0:
            continue                                                          # (after the cut alone the means are those of before)
        Q = np.zeros((2, hk, 1, d))
        Q[..., 0] = 1
        Q = bf16(Q + rng.normal(size=Q.shape) * 2.0 ** -4)
        idx, kept = torch.zeros(2, hk, 1, 3, dtype=torch.int32, device=DEV), torch.zeros(2, hk, 1, dtype=torch.int32, device=DEV)
        rb.rsa_cache_select(cache, rb.make_rows(Q), Q, kv, None, 1, 2, 0, 0, rb.RSA_CACHE_CAUSAL, idx, kept)
        for (b, h, g), x in ref.select(f64(Q), held, None, 1, 2, 0, 0, True).items():
            assert int(kept[b, h, g]) == len(x) and idx[b, h, g].tolist() == x + [-1] * (3 - len(x))
            kept_blocks.append((sum(ct) > 4, (held[b] - 1) // block in x))
    assert all(last for many, last in kept_blocks if many) and not all(last for many, last in kept_blocks if not many)


@pytest.mark.parametrize("d,block,ws", [(64, 64, True), (128, 128, False)])
def test_causal_prompts_of_many_tiles(d, block, ws):
    """More workgroups than the chip takes at once, so that the last tokens go first: outputs and log-sum-exps of the first, middle and last tiles."""
    hk, G, t, n = 2, 8, 4120, 4200
    p = Pair(1, hk, d, block, -(-n // block))
    p.fill([n], spread=0.3)
    Q = bf16(video_like(p.rng, 1, hk * G, t, d))
    assert hk * -(-t * G // 128) > 2 * 256                         # tiles of 128 rows and compute units, twice
    O, lse, rows = torch.full_like(Q, 7.0), torch.full(Q.shape[:3], 7.0, device=DEV), rb.make_rows(Q)
    scratch = torch.empty(max(256, rb.rsa_fourbit_workspace_bytes(p.gpu, rows)), dtype=torch.uint8, device=DEV) if ws else None
    rb.rsa_fourbit_attn(p.gpu, rows, Q, i32([n]), None, 0.0, rb.RSA_CACHE_CAUSAL, None, None, 0, O, lse, scratch)
    for i in (0, 1, 15, 16, 17, t // 2 - 1, t // 2, t - 25, t - 24, t - 9, t - 8, t - 1):
        ref = p.ref.attend(f64(Q[:, :, i:i + 1]), [n - t + i + 1], None, 0.0, False)
        compare(f64(O[:, :, i:i + 1]), lse[:, :, i:i + 1].cpu().double().numpy(), ref, d)
