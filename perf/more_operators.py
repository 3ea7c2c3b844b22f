"""Operators around a paged key/value cache as cases that can be timed and compared: what stands between the lengths of the
requests and the attention outputs, with the cache held in 4 bits.

  assign   rsa_cache_assign: pages for the new tokens of every sequence, with their positions and slots, from the lengths alone
  rotary   rsa_rotary_apply: queries and keys turned by their positions, or gradients turned back
  store    rsa_fourbit_write, rsa_fourbit_read: new keys and values into the pages, and back in bf16
  attn     rsa_fourbit_attn: attention of new queries over the cache, all of it or listed blocks

A code of the cache is e2m1 (sign, 0 0.5 1 1.5 2 3 4 6) over a power of two: one for each 32 channels of a key, one for each
value row. Shapes are those of ``synth.CONFIGS`` (a frame of 30 x 52 or 45 x 80 tokens, clips of 20 280 to 119 056 tokens, 24
heads, blocks of 64 and 128, 90 % sparsity) and generic ones of token-by-token decoding. Without ``own`` an operator is computed
by elementary torch operations in 32 bits (angles, and sums that decide on a rounding, in 64).
"""
import math

import torch

own = False

F32, F64, I64, BF16, U8 = torch.float32, torch.float64, torch.int64, torch.bfloat16, torch.uint8
GRID = (45, 80)                    # tokens of a frame, for positions along three axes


# ---- cases ---------------------------------------------------------------------------------------
def _case(kind, batch, heads, heads_kv, head_dim, block, t, kv, ragged=False, causal=False, group=0, keep=0, first=0, last=0,
          layout="bhtd", short=False, rot=0, pairing="half", axes=1, scaled="none", inverse=False):
    return {"kind": kind, "batch": batch, "heads": heads, "heads_kv": heads_kv, "head_dim": head_dim, "block": block, "t": t, "kv": kv,
            "ragged": ragged, "causal": causal, "group": group, "keep": keep, "first": first, "last": last, "layout": layout,
            "short": short, "rot": rot, "pairing": pairing, "axes": axes, "scaled": scaled, "inverse": inverse}


def listed():
    return [
        # one decoding step of 32 sequences: where each new token goes, a new page where the last one is full
        dict(_case("assign", 32, 8, 8, 128, 64, 1, 32768, ragged=True), name="assign_token"),
        # 48 prompts enter an empty cache together
        dict(_case("assign", 48, 8, 8, 128, 128, 4096, 4096, ragged=True), name="assign_prompts"),
        # one decoding step: query and key of each sequence, half of the channels, frequencies for a context that was lengthened
        dict(_case("rotary", 32, 32, 8, 128, 64, 1, 32768, ragged=True, rot=64, scaled="parts"), name="rotary_token"),
        # a 720p clip with its prompt, turned along time, height and width
        dict(_case("rotary", 1, 24, 24, 128, 128, 119056, 119056, layout="bthd", rot=128, pairing="interleaved", axes=3), name="rotary_clip"),
        # the gradient of three sequences of narrow heads, the whole head
        dict(_case("rotary", 3, 12, 12, 64, 64, 2077, 20280, ragged=True, rot=64, scaled="linear", inverse=True), name="rotary_gradient"),
        # one decoding step: the new token of each of 8 sequences goes into its half full block and comes back as attention sees it
        dict(_case("store", 8, 8, 8, 128, 64, 1, 4096, ragged=True), name="store_token"),
        # three sequences of different length and narrow heads, an odd number of tokens
        dict(_case("store", 3, 12, 12, 64, 64, 2077, 2077, ragged=True), name="store_ragged"),
        # a whole 720p clip with its prompt enters the cache at once and is read for the entry points that take bf16
        dict(_case("store", 1, 24, 24, 128, 128, 119056, 119056, layout="bthd"), name="store_clip"),
        # the smallest call: three drafted tokens on a short cache
        dict(_case("attn", 1, 2, 2, 64, 64, 3, 1088, causal=True), name="attn_draft"),
        # decoding of 32 sequences of different length, four query heads to a key/value head
        dict(_case("attn", 32, 32, 8, 128, 64, 1, 32768, ragged=True, causal=True), name="attn_token_batch"),
        # a new 30 x 52 frame sees the whole short clip
        dict(_case("attn", 1, 24, 24, 128, 128, 1560, 20280, layout="bthd"), name="attn_frame"),
        # a new 45 x 80 frame, 93 of 929 blocks for every 128 tokens
        dict(_case("attn", 1, 24, 24, 128, 128, 3600, 118800, group=128, keep=93, last=1, layout="bthd"), name="attn_frame_lists"),
    ]


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 200.0


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(["assign", "rotary", "rotary", "store", "attn", "attn", "attn"])
        head_dim, block = rng.choice([(128, 128), (128, 64), (64, 128), (64, 64)])
        batch = _log_int(rng, 1, 48)
        heads_kv = rng.choice([1, 2, 3, 8, 12, 24])
        heads = heads_kv * (rng.choice([1, 1, 2, 4, 5, 8]) if kind in ("rotary", "attn") else 1)
        kv = _log_int(rng, 1, 240000)
        t = rng.choice([1, 1, rng.randint(1, 8), _log_int(rng, 1, 4000), _log_int(rng, 100, 4000)])
        if kind in ("rotary", "store"):
            t = rng.choice([t, kv])
        t = min(t, kv)
        case = _case(kind, batch, heads, heads_kv, head_dim, block, t, kv, ragged=batch > 1 and rng.random() < 0.6,
                     causal=kind == "attn" and rng.random() < 0.5, layout=rng.choice(["bhtd", "bthd"]))
        blocks = -(-kv // block)
        if kind == "assign":
            case["short"] = rng.random() < 0.3
        if kind == "rotary":
            axes = rng.choice([1, 1, 1, 3])
            case.update(axes=axes, pairing=rng.choice(["half", "interleaved"]), inverse=rng.random() < 0.4, scaled=rng.choice(["none", "linear", "base", "parts"]),
                        rot=rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(6, head_dim // 2)]))
        if kind == "attn" and rng.random() < 0.4:
            # few blocks or up to a third of them; groups of one token while there are few, of 16 to 128 for frames
            case.update(group=1 if t <= 8 else rng.choice([16, 50, 64, 128]), keep=rng.randint(1, max(1, blocks // rng.choice([3, 10, 20]))),
                        first=rng.choice([0, 1]), last=rng.choice([1, 2]))
        if blocks > 16384 or heads > 96 or batch * heads * t > 24 * 240000 or batch * heads_kv * kv * head_dim > 24 * 237600 * 128:
            continue
        if kind == "attn" and batch * heads * t > 24 * 4000:
            continue
        if kind == "attn" and not case["group"] and batch * heads * t * kv > 24 * 1560 * 20280:
            continue
        if kind == "attn" and case["group"] and batch * heads_kv * -(-t // case["group"]) * _list_len(case) * block > 24 * 29 * 93 * 128:
            continue
        if _cost(case) <= most[kind]:
            return case


def _lengths(case):
    """(tokens in the cache, new or query tokens) of each sequence: ragged ones from all down to a quarter."""
    b, kv, t = case["batch"], case["kv"], case["t"]
    lens, rows = [], []
    for i in range(b):
        r = t - (i % 3) * (t // 4) if case["ragged"] else t
        n = kv - ((i * 7) % b) * (3 * kv // 4) // b if case["ragged"] else kv
        lens.append(max(n, r))
        rows.append(r)
    return lens, rows


def _list_len(case):
    blocks = -(-case["kv"] // case["block"])
    return min(blocks, max(case["keep"], case["first"] + case["last"] + -(-case["group"] // case["block"]) + 1))


def work(case):
    lens, rows = _lengths(case)
    hk, h, d, B, t = case["heads_kv"], case["heads"], case["head_dim"], case["block"], case["t"]
    token = d + d / 32 + 2                                 # bytes of a cached key and value
    byt = flops = 0.0
    for n, r in zip(lens, rows):
        if case["kind"] == "assign":
            # lengths in, lengths, start and count out; the new entries from the free list; a position and a slot for each row
            byt += 8 + 12 + 8 * (-(-n // B) - -(-(n - r) // B)) + 12 * t
            flops += 4.0 * t
        elif case["kind"] == "rotary":
            byt += (h + hk) * r * d * 4 + 4 * case["axes"] * r
            flops += 6.0 * (h + hk) * r * case["rot"] / 2
        elif case["kind"] == "store":
            # rows in, codes out; of the block that was begun before the keys' codes, for the mean; means; codes in, rows out
            byt += hk * (r * (d * 8 + 2 * token) + (n - r) % B * (d / 2 + d / 32) + (r / B + 1) * (4 + d))
            flops += 6.0 * hk * r * d
        else:
            keys = float(n)
            if case["group"]:
                keys = min(keys, float(_list_len(case)) * B)
                total = h * r * keys
                once = min(float(n), -(-r // case["group"]) * keys) * hk
            else:
                total = h * (r * keys - (r * (r - 1) / 2.0 if case["causal"] else 0.0))
                once = hk * keys
            byt += once * token + h * r * (d * 4 + 4)
            flops += 4.0 * total * d
    return {"bytes": byt, "flops": flops}


# ---- codes and pages, in torch -------------------------------------------------------------------
def _exponent(amax, largest, least):
    """The least e >= `least` with amax <= largest * 2^e."""
    m, e = torch.frexp(amax)
    lm, le = math.frexp(largest)
    return torch.where(amax > 0, (e - le + (m > lm).to(e.dtype)), torch.full_like(e, least)).clamp(min=least)


def _finite(x):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x))


def _quantise(x, run):
    """fp32 [..., d] in runs of `run` channels: e2m1 codes [..., d] and exponents [..., d / run]; a run with a value that is not
    finite has codes 0 and the exponent 128."""
    y = x.reshape(*x.shape[:-1], -1, run)
    bad = ~torch.isfinite(y).all(-1)
    e = _exponent(_finite(y).abs().amax(-1), 6.0, -124)
    z = torch.ldexp(y, -e[..., None])
    a = z.abs()
    # halves below 2, ones below 4, twos above; ties to the even code
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, 7.0))
    code = code.nan_to_num(0.0).to(U8) | (torch.signbit(z).to(U8) << 3)
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    return code.reshape(x.shape), torch.where(bad, torch.full_like(e, 128), e)


def _power(e):
    """2^e in fp32, NaN for the exponent 128."""
    return torch.where(e == 128, torch.full(e.shape, math.nan, device=e.device), torch.ldexp(torch.ones(e.shape, device=e.device), e.clamp(max=127)))


def _value(code):
    m = (code & 7).to(F32)
    a = torch.where(m <= 4, m / 2, torch.where(m <= 6, m - 2, 6.0))
    return torch.where(code >= 8, -a, a)


def _pairs(x):
    return x[..., 0::2] | (x[..., 1::2] << 4)


def _unpairs(x):
    return torch.stack([x & 15, x >> 4], -1).flatten(-2)


def _pack_k(code, e):
    """codes [..., B, d], exponents [..., B, d/32] -> bytes: for 64 keys four pieces of 16, in them (32 channels, key, 16 bytes); then the
    exponents + 127 as (32 channels, key of 16, piece)."""
    lead, (B, d), n = code.shape[:-2], code.shape[-2:], code.dim() - 2
    a = _pairs(code).reshape(*lead, B // 64, 4, 16, d // 32, 16).permute(*range(n + 2), n + 3, n + 2, n + 4).reshape(*lead, B // 64, 32 * d)
    s = (e + 127).to(U8).reshape(*lead, B // 64, 4, 16, d // 32).permute(*range(n + 1), n + 3, n + 2, n + 1).reshape(*lead, B // 64, 2 * d)
    return torch.cat([a, s], -1).flatten(-2)


def _unpack_k(x, B, d):
    lead, n = x.shape[:-1], x.dim() - 1
    x = x.reshape(*lead, B // 64, 34 * d)
    a = x[..., :32 * d].reshape(*lead, B // 64, 4, d // 32, 16, 16).permute(*range(n + 2), n + 3, n + 2, n + 4).reshape(*lead, B, d // 2)
    s = x[..., 32 * d:].reshape(*lead, B // 64, d // 32, 16, 4).permute(*range(n + 1), n + 3, n + 2, n + 1).reshape(*lead, B, d // 32)
    return _unpairs(a), s.to(torch.int32) - 127


def _pack_v(code, e):
    """codes [..., B, d], exponents [..., B] -> bytes: for 64 keys (32 channels, g, channel of 16, half, t, i), key 16 t + 4 g + i; then the scales in
    bf16 as (g, t, i)."""
    lead, (B, d), n = code.shape[:-2], code.shape[-2:], code.dim() - 2
    a = code.reshape(*lead, B // 64, 4, 4, 4, d // 32, 2, 16)                            # t, g, i, c, half, channel
    a = _pairs(a.permute(*range(n + 1), n + 4, n + 2, n + 6, n + 5, n + 1, n + 3).reshape(*lead, B // 64, 64 * d))
    s = _power(e).to(BF16).reshape(*lead, B // 64, 4, 4, 4).transpose(-3, -2).reshape(*lead, B // 64, 64)
    return torch.cat([a, s.contiguous().view(U8)], -1).flatten(-2)


def _unpack_v(x, B, d):
    """codes [..., B, d] and scales in fp32 [..., B]"""
    lead, n = x.shape[:-1], x.dim() - 1
    x = x.reshape(*lead, B // 64, 32 * d + 128)
    a = _unpairs(x[..., :32 * d]).reshape(*lead, B // 64, d // 32, 4, 16, 2, 4, 4)       # c, g, channel, half, t, i
    a = a.permute(*range(n + 1), n + 5, n + 2, n + 6, n + 1, n + 4, n + 3).reshape(*lead, B, d)
    s = x[..., 32 * d:].contiguous().view(BF16).reshape(*lead, B // 64, 4, 4, 4).transpose(-3, -2).reshape(*lead, B)
    return a, s.to(F32)


def _keys_of(x, B, d):
    code, e = _unpack_k(x, B, d)
    return (_value(code).unflatten(-1, (-1, 32)) * _power(e)[..., None]).flatten(-2)


def _values_of(x, B, d):
    code, s = _unpack_v(x, B, d)
    return _value(code) * s[..., None]


def _mean_codes(k, n):
    """int8 codes and exponents of the mean of the first n rows of k [..., B, d] (zeros behind them)."""
    mean = _finite(k).to(F64).sum(-2) / n.clamp(min=1).unsqueeze(-1)
    e = _exponent(mean.abs().amax(-1), 127.0, -100)
    return torch.round(torch.ldexp(mean, -e.unsqueeze(-1))).to(torch.int8), e


# ---- inputs --------------------------------------------------------------------------------------
def _smooth(gen, heads, tokens, d, noise):
    """Neighbouring tokens are alike, as those of a video are: four slow waves for each channel, and noise; [heads, tokens, d]."""
    f = torch.rand(heads, 4, 1, generator=gen, device="cuda") * 60 + 3
    pos = torch.arange(tokens, device="cuda", dtype=F32) / 120000.0
    amp = torch.randn(2, heads, 4, d, generator=gen, device="cuda") * 0.5
    x = (torch.randn(heads, tokens, d, generator=gen, device="cuda") * noise)
    theta = 2 * math.pi * f * pos
    x += torch.matmul(torch.sin(theta).transpose(1, 2).contiguous(), amp[0]) + torch.matmul(torch.cos(theta).transpose(1, 2).contiguous(), amp[1])
    return x


def _as_layout(x, layout):
    x = x.to(BF16)
    return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if layout == "bthd" else x.contiguous()


def _axis_pairs(case):
    """Pairs of channels that turn along each axis: a sixth and the rest in two for time, height and width."""
    n = case["rot"] // 2
    if case["axes"] == 1:
        return [n]
    a = max(1, n // 8)
    return [a, (n - a + 1) // 2, (n - a) // 2]


def _frequencies(case):
    """Radians a position of each pair, fp64, and what the outputs are multiplied by."""
    freq, factor = [], 1.0
    for n in _axis_pairs(case):
        base = 10000.0 if case["axes"] == 3 else 500000.0
        if case["scaled"] == "base" and n > 1:
            base *= 8.0 ** (n / (n - 1.0))
        f = [base ** (-j / n) for j in range(n)]
        if case["scaled"] == "linear":
            f = [x / 4.0 for x in f]
        if case["scaled"] == "parts":
            # frequencies that turn often within the old length stay, those that do not turn once are stretched
            factor = 0.1 * math.log(8.0) + 1.0
            keep = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
            f = [x * (k + (1 - k) / 8.0) for x, k in zip(f, keep)]
        freq += f
    return freq, factor


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    b, h, hk, d, B, t = (case[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t"))
    lens, rows = _lengths(case)
    i32 = dict(dtype=torch.int32, device="cuda")
    s = {"case": case, "kv_len": torch.tensor(lens, **i32), "q_len": torch.tensor(rows, **i32)}
    s["start"] = s["kv_len"] - s["q_len"]
    if case["kind"] == "rotary":
        freq, s["factor"] = _frequencies(case)
        s["freq"] = torch.tensor(freq, dtype=F64, device="cuda")
        if case["axes"] == 3:
            at = s["start"].long()[:, None] + torch.arange(t, device="cuda")
            s["positions"] = torch.stack([at // (GRID[0] * GRID[1]), at // GRID[1] % GRID[0], at % GRID[1]]).to(torch.int32).contiguous()
        for name, n in (("Q", h), ("K", hk)):
            s[name] = _as_layout(torch.randn(b, n, t, d, generator=gen, device="cuda"), case["layout"])
            s[name + "r"] = torch.zeros_like(s[name])
        return s
    held = [n - r for n, r in zip(lens, rows)] if case["kind"] in ("assign", "store") else lens
    blocks = [-(-n // B) for n in lens]
    old = [-(-n // B) for n in held] if case["kind"] == "assign" else blocks
    width, pages = max(blocks), sum(blocks) + 3
    table = torch.full((b, width), -1, dtype=torch.int32)
    # pages are handed out in no order; the last one never
    order = torch.randperm(pages - 1, generator=torch.Generator().manual_seed(int(seed) + 1)).to(torch.int32)
    at = 0
    for i, n in enumerate(old):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"] = table.cuda()
    if case["kind"] == "assign":
        free = order[at:]
        s["free_pages"] = torch.zeros(pages, dtype=torch.int32)
        s["free_pages"][:len(free)] = free
        s["free_pages"] = s["free_pages"].cuda()
        # with too few pages the last sequences get none
        s["free_count"] = torch.tensor([len(free) // 2 if case["short"] else len(free)], **i32)
        s["kv_len"], s["add"] = s["start"], s["q_len"]
        s["out"] = {"kv_new": torch.zeros(b, **i32), "free_left": torch.zeros(1, **i32), "start": torch.zeros(b, **i32), "count": torch.zeros(b, **i32),
                    "positions": torch.zeros(b, t, **i32), "slots": torch.zeros(b, t, dtype=I64, device="cuda")}
        return s
    s["k_codes"] = torch.zeros(pages, hk, B * (d // 2 + d // 32), dtype=U8, device="cuda")
    s["v_codes"] = torch.zeros(pages, hk, B * (d // 2 + 2), dtype=U8, device="cuda")
    s["scales"], s["k_mean"] = torch.zeros(pages, hk, 4, dtype=F32, device="cuda"), torch.zeros(pages, hk, d, dtype=torch.int8, device="cuda")
    for i, n in enumerate(held):
        nb = -(-n // B)
        for lo in range(0, nb, 256):                     # (some blocks at a time)
            m = min(256, nb - lo)
            page = s["table"][i, lo:lo + m].long()
            left = (n - (lo + torch.arange(m, device="cuda")) * B).clamp(max=B)
            there = (torch.arange(B, device="cuda") < left[:, None])[:, None, :, None]
            for which in ("k", "v"):
                x = _smooth(gen, hk, m * B, d, 0.5) if which == "k" else torch.randn(hk, m * B, d, generator=gen, device="cuda")
                x = x.to(BF16).to(F32).reshape(hk, m, B, d).transpose(0, 1)
                x = torch.where(there, x, torch.zeros_like(x))
                code, e = _quantise(x, 32 if which == "k" else d)
                s[which + "_codes"][page] = _pack_k(code, e) if which == "k" else _pack_v(code, e[..., 0])
                if which == "k":
                    k = (_value(code).unflatten(-1, (-1, 32)) * _power(e)[..., None]).flatten(-2)
                    mean, em = _mean_codes(k, left[:, None].expand(m, hk))
                    s["k_mean"][page] = mean
                    s["scales"][page, :, 2] = torch.ldexp(torch.ones_like(em, dtype=F32), em)
    if case["kind"] == "store":
        s["K"] = _as_layout(torch.stack([_smooth(gen, hk, t, d, 0.5) for _ in range(b)]), case["layout"])
        s["V"] = _as_layout(torch.randn(b, hk, t, d, generator=gen, device="cuda"), case["layout"])
        s["Kb"], s["Vb"] = torch.zeros_like(s["K"]), torch.zeros_like(s["V"])
        return s
    s["Q"] = _as_layout(torch.stack([_smooth(gen, h, t, d, 0.5) for _ in range(b)]), case["layout"])
    if case["group"]:
        s["block_idx"], s["kept"] = _choose(s)           # the lists are an input here
    s["O"] = torch.zeros_like(s["Q"])
    s["lse"] = torch.zeros(b, h, t, dtype=F32, device="cuda")
    return s


def _choose(s):
    """Lists as the framework's selection leaves them: forced blocks and, by the score of their mean keys, the best others."""
    c = s["case"]
    b, h, hk, d, B, t, group = (c[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t", "group"))
    groups, L, M = -(-t // group), _list_len(c), s["table"].shape[1]
    kv, r = s["kv_len"].long(), s["q_len"].long()
    q = torch.where((torch.arange(t, device="cuda") < r[:, None])[:, None, :, None], s["Q"].to(F32), 0.0)
    q = _group_rows(q, group).reshape(b, hk, h // hk, groups, group, d).sum((2, 4))
    safe = s["table"].long().clamp(min=0)
    mean = (s["k_mean"][safe].to(F32) * s["scales"][safe][..., 2:3]).transpose(1, 2)
    score = torch.matmul(q, mean.transpose(-1, -2).contiguous())
    lo = torch.arange(groups, device="cuda") * group
    first = (kv - r)[:, None] + lo
    last = (kv - r)[:, None] + torch.minimum(lo + group, r[:, None]) - 1
    blk = torch.arange(M, device="cuda")
    seen = torch.where(torch.full_like(last, c["causal"], dtype=torch.bool), last // B + 1, ((kv + B - 1) // B)[:, None])
    visible = (blk < seen[..., None]) & (lo < r[:, None])[..., None]
    forced = (blk < c["first"]) | ((blk > (first // B)[..., None] - c["last"]) & (blk <= (last // B)[..., None]) & (c["last"] > 0))
    score = torch.where(forced[:, None], torch.full_like(score, math.inf), score)
    score = torch.where(visible[:, None], score, torch.full_like(score, -math.inf))
    place = torch.argsort(torch.argsort(score, dim=-1, descending=True, stable=True), dim=-1, stable=True)
    kept = (place < (visible & forced).sum(-1).clamp(min=c["keep"])[:, None, :, None]) & visible[:, None]
    idx = torch.where(kept, blk.expand_as(kept), torch.full_like(blk, M).expand_as(kept)).sort(-1).values[..., :L]
    return torch.where(idx < M, idx, torch.full_like(idx, -1)).to(torch.int32).contiguous(), kept.sum(-1).to(torch.int32)


# ---- the plain forms -----------------------------------------------------------------------------
def _assign(s):
    c, o = s["case"], s["out"]
    b, B, t, M = c["batch"], c["block"], c["t"], s["table"].shape[1]
    held, add = s["kv_len"].long().clamp(0, M * B), s["add"].long().clamp(0, t)
    want = held + add
    had, need = -(-held // B), -(-want // B)
    free = s["free_count"].long().clamp(0, s["free_pages"].shape[0])
    more = torch.where(want <= M * B, need - had, torch.zeros_like(need))
    upto = more.cumsum(0)
    granted = (want <= M * B) & ((more == 0) | (upto <= free))
    taken = torch.where(granted, more, torch.zeros_like(more))
    blk = torch.arange(M, device="cuda")
    at = free - 1 - (upto - more)[:, None] - (blk - had[:, None])
    new = (blk >= had[:, None]) & (blk < (had + taken)[:, None])
    s["table"].copy_(torch.where(new, s["free_pages"][at.clamp(0, s["free_pages"].shape[0] - 1)], s["table"]))
    count = torch.where(granted, add, torch.zeros_like(add))
    o["kv_new"].copy_(held + count)
    o["free_left"].copy_(free - taken.sum())
    o["start"].copy_(held)
    o["count"].copy_(count)
    i = torch.arange(t, device="cuda")
    pos, there = held[:, None] + i, i < count[:, None]
    page = torch.gather(s["table"].long(), 1, (pos // B).clamp(max=M - 1))
    o["positions"].copy_(torch.where(there, pos, -1))
    o["slots"].copy_(torch.where(there & (page >= 0), page * B + pos % B, -1))


def _rotary(s):
    c = s["case"]
    t, n = c["t"], c["rot"] // 2
    if c["axes"] == 1:
        pos = (s["start"].to(F64)[:, None] + torch.arange(t, device="cuda"))[..., None]                  # [b, t, 1]
    else:
        pos = torch.repeat_interleave(s["positions"].to(F64), torch.tensor(_axis_pairs(c), device="cuda"), dim=0).permute(1, 2, 0)
    angle = (pos * s["freq"])[:, None]                                                                   # [b, 1, t, n]
    cos, sin = (torch.cos(angle) * s["factor"]).to(F32), (torch.sin(angle) * s["factor"]).to(F32)
    if c["inverse"]:
        sin = -sin
    mine = (torch.arange(t, device="cuda") < s["q_len"].long()[:, None])[:, None, :, None]
    for name in ("Q", "K"):
        x = s[name].to(F32)
        a, z = (x[..., :n], x[..., n:2 * n]) if c["pairing"] == "half" else (x[..., :2 * n:2], x[..., 1:2 * n:2])
        y = torch.stack([a * cos - z * sin, a * sin + z * cos], -2 if c["pairing"] == "half" else -1).flatten(-2)
        y = torch.cat([y, x[..., 2 * n:]], -1).to(BF16)
        s[name + "r"].copy_(torch.where(mine, y, s[name + "r"]))


def _store(s):
    c = s["case"]
    b, hk, d, B, t = (c[k] for k in ("batch", "heads_kv", "head_dim", "block", "t"))
    M = s["table"].shape[1]
    J = min((t - 1) // B + 2, M)
    start, count = s["start"].long(), s["q_len"].long()
    blk = (start // B).clamp(max=M - J)[:, None] + torch.arange(J, device="cuda")        # [b, J]
    page = torch.gather(s["table"].long(), 1, blk)
    pos = blk[..., None] * B + torch.arange(B, device="cuda")                            # [b, J, B]
    new = (pos >= start[:, None, None]) & (pos < (start + count)[:, None, None])
    touched = new.any(-1) & (page >= 0)
    n = torch.where(new, pos % B + 1, torch.zeros_like(pos)).amax(-1)                    # tokens that the block holds then
    safe = torch.where(page >= 0, page, torch.full_like(page, s["k_codes"].shape[0] - 1))
    row = (pos - start[:, None, None]).clamp(0, t - 1).reshape(b, 1, J * B, 1).expand(b, hk, J * B, d)
    fresh, there = new[:, :, None, :, None], touched[:, :, None]
    take = lambda X: torch.gather(X, 2, row).reshape(b, hk, J, B, d).transpose(1, 2).to(F32)      # [b, J, hk, B, d]
    code, e = _quantise(take(s["K"]), 32)
    was = s["k_codes"][safe]
    code_was, e_was = _unpack_k(was, B, d)
    code, e = torch.where(fresh, code, code_was), torch.where(fresh, e, e_was)
    s["k_codes"][safe] = torch.where(there[..., None], _pack_k(code, e), was)
    k = (_value(code).unflatten(-1, (-1, 32)) * _power(e)[..., None]).flatten(-2)
    held = (torch.arange(B, device="cuda") < n[..., None])[:, :, None, :, None]
    mean, em = _mean_codes(torch.where(held, k, torch.zeros_like(k)), n[:, :, None].expand(b, J, hk))
    s["k_mean"][safe] = torch.where(there[..., None], mean, s["k_mean"][safe])
    s["scales"][..., 2][safe] = torch.where(there, torch.ldexp(torch.ones_like(em, dtype=F32), em), s["scales"][..., 2][safe])
    del code, e, code_was, e_was, k
    code, e = _quantise(take(s["V"]), d)
    was = s["v_codes"][safe]
    code_was, scale_was = _unpack_v(was, B, d)
    code = torch.where(fresh, code, code_was)
    e = torch.where(fresh[..., 0], e[..., 0], torch.where(torch.isnan(scale_was), 128, torch.frexp(scale_was)[1] - 1))
    s["v_codes"][safe] = torch.where(there[..., None], _pack_v(code, e), was)
    del code, e, code_was, scale_was
    # and the range back
    pos = start[:, None] + torch.arange(t, device="cuda")
    mine = (torch.arange(t, device="cuda") < count[:, None])[:, None, :, None]
    at = pos.clamp(max=M * B - 1)[:, None, :, None].expand(b, hk, t, d)
    page = s["table"].long().clamp(min=0)
    for codes, values, X in ((s["k_codes"], _keys_of, s["Kb"]), (s["v_codes"], _values_of, s["Vb"])):
        x = values(codes[page], B, d).transpose(1, 2).reshape(b, hk, -1, d)
        X.copy_(torch.where(mine, torch.gather(x, 2, at).to(BF16), X))


def _group_rows(x, group):
    """[b, h, t, ...] -> [b, h, groups, group, ...], zeros behind."""
    t = x.shape[2]
    groups = -(-t // group)
    full = torch.zeros(*x.shape[:2], groups * group, *x.shape[3:], dtype=x.dtype, device=x.device)
    full[:, :, :t] = x
    return full.reshape(*x.shape[:2], groups, group, *x.shape[3:])


def _softmax_rows(q, k, v, seen):
    """q [..., r, d], k and v [..., n, d], seen [..., r, n]: outputs and log-sum-exp, 0 and -inf for a row that sees nothing."""
    a = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(q.shape[-1]))
    a = torch.where(seen, a, torch.full_like(a, -math.inf))
    m = a.amax(-1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    p = torch.exp(a - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (torch.log(total) + m).squeeze(-1)


def _attn(s):
    c = s["case"]
    b, h, hk, d, B, t, group = (c[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t", "group"))
    per = group or t
    groups = -(-t // per)
    q = _group_rows(s["Q"].to(F32), per).reshape(b, hk, h // hk, groups, per, d).transpose(2, 3)
    q = q.reshape(b, hk, groups, h // hk * per, d)                                        # [b, hk, groups, G * per, d]
    if group:
        blk = s["block_idx"].long()                                                       # [b, hk, groups, L]
        page = torch.where(blk >= 0, torch.gather(s["table"].long()[:, None, None].expand(b, hk, groups, -1), 3, blk.clamp(min=0)), -1)
        head = torch.arange(hk, device="cuda")[None, :, None, None].expand_as(page)
        k, v = (f(s[name][page.clamp(min=0), head], B, d).reshape(b, hk, groups, -1, d) for f, name in ((_keys_of, "k_codes"), (_values_of, "v_codes")))
    else:
        page = s["table"].long()[:, None, None]
        blk = torch.arange(page.shape[-1], device="cuda").expand(b, 1, 1, -1)
        k, v = (f(s[name][page[:, 0, 0].clamp(min=0)], B, d).transpose(1, 2).reshape(b, hk, 1, -1, d) for f, name in ((_keys_of, "k_codes"), (_values_of, "v_codes")))
    key = (blk[..., None] * B + torch.arange(B, device="cuda")).flatten(-2)               # [b, hk|1, groups|1, n]
    there = (page >= 0)[..., None].expand(*page.shape, B).flatten(-2) & (key >= 0)
    kv, r = s["kv_len"].long(), s["q_len"].long()
    row = torch.arange(groups * per, device="cuda").reshape(groups, per).repeat(1, h // hk)            # [groups, G * per]
    bound = (kv - r)[:, None, None] + row + 1 if c["causal"] else kv[:, None, None].expand(b, *row.shape)
    seen = there[..., None, :] & (key[..., None, :] < torch.minimum(bound, kv[:, None, None])[:, None, :, :, None])
    o, lse = _softmax_rows(q, k, v, seen)
    back = lambda x: x.reshape(b, hk, groups, h // hk, per, *x.shape[4:]).transpose(2, 3).reshape(b, h, groups * per, *x.shape[4:])[:, :, :t]
    mine = (torch.arange(t, device="cuda") < r[:, None])[:, None]
    s["O"].copy_(torch.where(mine[..., None], back(o).to(BF16), s["O"]))
    s["lse"].copy_(torch.where(mine, back(lse), s["lse"]))


# ---- one pass ------------------------------------------------------------------------------------
def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "assign":
        return {"table": s["table"], **s["out"]}
    if kind == "rotary":
        return {"q": s["Qr"], "k": s["Kr"]}
    if kind == "store":
        return {"k": s["Kb"], "v": s["Vb"], "mean": s["k_mean"], "mean_scale": s["scales"][..., 2]}
    return {"o": s["O"], "lse": s["lse"]}


def _records(s, rb):
    """The records that a program makes once for its cache and its tensors."""
    c = s["case"]
    if c["kind"] == "assign":
        s["pages"] = rb.pages_of(s["table"], s["free_pages"], c["block"])
    elif c["kind"] == "rotary":
        s["rotary"] = rb.make_rotary(s["freq"], c["pairing"], _axis_pairs(c), s["factor"])
        s["rows"], s["rows_k"] = rb.make_rows(s["Q"]), rb.make_rows(s["K"])
    else:
        s["cache"] = rb.fourbit_of(s["k_codes"], s["v_codes"], s["scales"], s["k_mean"], s["table"], c["block"])
        s["rows"] = rb.make_rows(s["K"] if "K" in s else s["Q"])
        if c["kind"] == "attn":
            s["ws"] = torch.empty(max(256, rb.rsa_fourbit_workspace_bytes(s["cache"], s["rows"], c["group"])), dtype=U8, device="cuda")
    s["made"] = True


def _run_own(s):
    from paper_2511_19835_amd import binding as rb
    c = s["case"]
    if "made" not in s:
        _records(s, rb)
    if c["kind"] == "assign":
        o = s["out"]
        rb.rsa_cache_assign(s["pages"], c["t"], s["kv_len"], s["add"], s["free_count"], o["kv_new"], o["free_left"], o["start"], o["count"],
                            o["positions"], o["slots"])
    elif c["kind"] == "rotary":
        rb.rsa_rotary_apply(s["rotary"], s["rows"], s["Q"], s["Qr"], s["rows_k"], s["K"], s["Kr"], s.get("positions"), s["start"], s["q_len"],
                            rb.RSA_ROTARY_INVERSE if c["inverse"] else 0)
    elif c["kind"] == "store":
        rb.rsa_fourbit_write(s["cache"], s["rows"], s["K"], s["V"], s["start"], s["q_len"])
        rb.rsa_fourbit_read(s["cache"], s["rows"], s["start"], s["q_len"], s["Kb"], s["Vb"])
    else:
        rb.rsa_fourbit_attn(s["cache"], s["rows"], s["Q"], s["kv_len"], s["q_len"], 0.0, rb.RSA_CACHE_CAUSAL if c["causal"] else 0, s.get("block_idx"),
                            s.get("kept"), c["group"], s["O"], s["lse"], s["ws"])


def run(s):
    if own:
        _run_own(s)
    else:
        {"assign": _assign, "rotary": _rotary, "store": _store, "attn": _attn}[s["case"]["kind"]](s)
    return _outputs(s)


# ---- the definitions in 64 bits ------------------------------------------------------------------
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest64(x):
    """fp64, |x| <= 6, to the nearest level; between two the one with the even number."""
    levels = torch.tensor(LEVELS, dtype=F64, device=x.device)
    a = x.abs()
    best = torch.zeros_like(a)
    for i in range(1, 8):
        mid = (LEVELS[i - 1] + LEVELS[i]) / 2
        best = torch.where((a > mid) | ((a == mid) & (i % 2 == 0)), levels[i], best)
    return torch.where(x < 0, -best, best)


def _stored64(x, run):
    """What is held of fp64 rows [..., d] in runs of `run` channels."""
    y = x.reshape(*x.shape[:-1], -1, run)
    amax = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -140) / 6.0)).clamp(min=-124.0)
    e = torch.where((amax <= 6.0 * torch.exp2(e - 1)) & (e > -124), e - 1, torch.where(amax > 6.0 * torch.exp2(e), e + 1, e))
    return (_nearest64(y / torch.exp2(e)) * torch.exp2(e)).reshape(x.shape)


def _places(B, d):
    """Half bytes of (token, channel) in a page's keys and values, and the places of their scales (bytes of keys, pairs of bytes of values)."""
    t, ch = torch.arange(B, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    u = t % 64
    k = t // 64 * (68 * d) + ((u // 16 * (d // 32) + ch // 32) * 16 + u % 16) * 32 + ch % 32
    ks = t // 64 * (34 * d) + 32 * d + (ch // 32 * 16 + u % 16) * 4 + u // 16
    v = t // 64 * (64 * d + 256) + ((ch // 32 * 4 + u % 16 // 4) * 16 + ch % 16) * 32 + ch % 32 // 16 * 16 + u // 16 * 4 + u % 4
    vs = t[:, 0] // 64 * (16 * d + 64) + 16 * d + u[:, 0] % 16 // 4 * 16 + u[:, 0] // 16 * 4 + u[:, 0] % 4
    return k, ks, v, vs


def _tokens64(s, i, j, lo, hi):
    """Keys and values of tokens lo..hi-1 of head j, sequence i, fp64 [hi - lo, d]."""
    c = s["case"]
    B, d, hk = c["block"], c["head_dim"], c["heads_kv"]
    tok = torch.arange(lo, hi, device="cuda")
    rec = (s["table"][i].long()[tok // B] * hk + j)[:, None]
    k, ks, v, vs = (x[tok % B] for x in _places(B, d))
    levels = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=F64, device="cuda")
    out = []
    for name, place, size in (("k_codes", k, B * (d // 2 + d // 32)), ("v_codes", v, B * (d // 2 + 2))):
        flat = s[name].reshape(-1)
        code = levels[(flat[rec * size + place // 2].long() >> (place % 2 * 4)) & 15]
        if name == "k_codes":
            e = flat[rec * size + ks].to(F64) - 127
            code = code * torch.exp2(e)
        else:
            bits = s[name].reshape(-1, 2)[rec[:, 0] * (size // 2) + vs].long()
            code = code * torch.exp2(((bits[:, 0] >> 7) + (bits[:, 1] & 127) * 2).to(F64) - 127)[:, None]
        out.append(code)
    return out


def _exact_assign(s):
    c = s["case"]
    b, B, t, M = c["batch"], c["block"], c["t"], s["table"].shape[1]
    table, held, add = s["table"].cpu().clone(), s["kv_len"].tolist(), s["add"].tolist()
    free, stack = int(s["free_count"]), s["free_pages"].tolist()
    start, count, wanted = [], [], 0
    pos, slot = torch.full((b, t), -1, dtype=torch.int32), torch.full((b, t), -1, dtype=I64)
    left = free
    for i in range(b):
        n = held[i] + add[i]
        more = max(0, -(-n // B) - -(-held[i] // B))
        fits = n <= M * B
        wanted += more if fits else 0
        ok = fits and (more == 0 or wanted <= free)
        if ok:
            for j in range(more):
                table[i, -(-held[i] // B) + j] = stack[free - 1 - (wanted - more) - j]
            left -= more
            p = torch.arange(held[i], n)
            pos[i, :add[i]] = p.to(torch.int32)
            slot[i, :add[i]] = table[i].long()[p // B] * B + p % B
        start.append(held[i])
        count.append(add[i] if ok else 0)
    as32 = lambda x: torch.tensor(x, dtype=torch.int32)
    return {"table": table, "kv_new": as32([x + y for x, y in zip(held, count)]), "free_left": as32([left]), "start": as32(start), "count": as32(count),
            "positions": pos, "slots": slot}


def _exact_rotary(s):
    c = s["case"]
    n, out = c["rot"] // 2, {}
    lens, rows = _lengths(c)
    for name, key in (("Q", "q"), ("K", "k")):
        y = torch.zeros(s[name].shape, dtype=F64, device="cuda")
        for i, r in enumerate(rows):
            at, angle = 0, []
            for axis, m in enumerate(_axis_pairs(c)):
                p = torch.arange(lens[i] - r, lens[i], device="cuda") if c["axes"] == 1 else s["positions"][axis, i, :r]
                angle.append(p.to(F64)[:, None] * s["freq"][at:at + m])
                at += m
            turn = torch.polar(torch.full((r, n), s["factor"], dtype=F64, device="cuda"), torch.cat(angle, 1) * (-1.0 if c["inverse"] else 1.0))
            for j in range(y.shape[1]):
                x = s[name][i, j, :r].to(F64)
                first, second = (slice(0, n), slice(n, 2 * n)) if c["pairing"] == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
                z = torch.complex(x[:, first], x[:, second]) * turn
                y[i, j, :r] = x
                y[i, j, :r, first], y[i, j, :r, second] = z.real, z.imag
        out[key] = y
    return out


def _exact_store(s):
    c = s["case"]
    hk, d, B = c["heads_kv"], c["head_dim"], c["block"]
    lens, rows = _lengths(c)
    if sum(-(-r // B) + 1 for r in rows) * hk > 6000:
        return None
    K, V = (torch.zeros(c["batch"], hk, c["t"], d, dtype=F64, device="cuda") for _ in range(2))
    mean, scale = s["k_mean"].clone(), s["scales"][..., 2].to(F64)
    for i, (n, r) in enumerate(zip(lens, rows)):
        K[i, :, :r], V[i, :, :r] = _stored64(s["K"][i, :, :r].to(F64), 32), _stored64(s["V"][i, :, :r].to(F64), d)
        for blk in range((n - r) // B, -(-n // B)):
            lo, hi, page = max(n - r, blk * B), min(n, blk * B + B), int(s["table"][i, blk])
            for j in range(hk):
                m = K[i, j, lo - (n - r):hi - (n - r)].sum(0)
                if lo > blk * B:
                    m = m + _tokens64(s, i, j, blk * B, lo)[0].sum(0)
                m = m / (hi - blk * B)
                amax, e = float(m.abs().max()), -100
                if amax > 0:
                    e = max(-100, math.floor(math.log2(amax / 127.0)) - 1)
                    while amax > math.ldexp(127.0, e):
                        e += 1
                mean[page, j], scale[page, j] = torch.round(m / 2.0 ** e).to(torch.int8), 2.0 ** e
    return {"k": K, "v": V, "mean": mean, "mean_scale": scale}


def _exact_attn(s):
    c = s["case"]
    h, hk, d, B, t, group = (c[k] for k in ("heads", "heads_kv", "head_dim", "block", "t", "group"))
    lens, rows = _lengths(c)
    G = h // hk
    if group and c["batch"] * hk * -(-t // group) > 3000:
        return None
    O = torch.zeros(c["batch"], h, t, d, dtype=F64, device="cuda")
    lse = torch.zeros(c["batch"], h, t, dtype=F64, device="cuda")
    tok = torch.arange(t, device="cuda")
    for i, (n, r) in enumerate(zip(lens, rows)):
        lists = s["block_idx"][i].cpu() if group else None
        for j in range(hk):
            k, v = _tokens64(s, i, j, 0, n)
            for g in range(-(-r // group) if group else 1):
                lo, hi = (g * group, min(r, g * group + group)) if group else (0, r)
                key = torch.arange(n, device="cuda")
                if group:
                    allowed = torch.zeros(-(-n // B), dtype=torch.bool, device="cuda")
                    allowed[[m for m in lists[j, g].tolist() if m >= 0]] = True
                    key = key[allowed[key // B]]
                q = s["Q"][i, j * G:j * G + G, lo:hi].to(F64).reshape(-1, d)
                a = torch.mm(q, k[key].t().contiguous()) * d ** -0.5
                if c["causal"]:
                    a.masked_fill_(key[None] > (n - r + tok[lo:hi]).repeat(G)[:, None], -math.inf)
                total = torch.logsumexp(a, 1)
                p = torch.exp(a - torch.where(torch.isfinite(total), total, 0.0)[:, None])
                O[i, j * G:j * G + G, lo:hi] = torch.mm(p, v[key]).reshape(G, hi - lo, d)
                lse[i, j * G:j * G + G, lo:hi] = total.reshape(G, hi - lo)
    return {"o": O, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"assign": _exact_assign, "rotary": _exact_rotary, "store": _exact_store, "attn": _exact_attn}[case["kind"]](s)
