"""The operators of the 8-bit key/value cache as cases that can be timed and compared.

A cache keeps the keys and values of earlier frames or tokens in pages of one block of tokens: e4m3 codes with a power-of-two
scale for each (page, key/value head), the order of the codes inside a page being the one in which the matrix instructions of the
attention take them, and an 8-bit mean of each page's keys. A case is one call of one of its operators:

  write    rsa_cache_write: new keys and values are quantised into the pages (and the means follow)
  read     rsa_cache_read: a range of tokens back in bf16
  select   rsa_cache_select: for every group of query tokens the blocks whose mean key scores best
  attn     rsa_cache_attn: attention of new queries over the cache, all of it or the listed blocks

Shapes are those of ``synth.CONFIGS`` (a frame of 30 x 52 or 45 x 80 tokens, clips of 20 280 to 119 056 tokens, 24 heads, blocks of
64 and 128, 90 % sparsity) and generic ones of token-by-token decoding. Without ``own`` an operator is computed by elementary torch
operations in 32 bits (sums that decide on a rounding or an order in 64).
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn
F32, F64, I64 = torch.float32, torch.float64, torch.int64


# ---- cases ---------------------------------------------------------------------------------------
def _case(kind, batch, heads, heads_kv, head_dim, block, t, kv, ragged=False, causal=False, group=0, keep=0, first=0, last=0,
          layout="bhtd"):
    return {"kind": kind, "batch": batch, "heads": heads, "heads_kv": heads_kv, "head_dim": head_dim, "block": block, "t": t, "kv": kv,
            "ragged": ragged, "causal": causal, "group": group, "keep": keep, "first": first, "last": last, "layout": layout}


def listed():
    return [
        # one decoding step: the new token of each of 8 sequences goes into its half full block
        dict(_case("write", 8, 8, 8, 128, 64, 1, 4096, ragged=True), name="write_token"),
        # a whole 720p clip with its prompt enters the cache at once
        dict(_case("write", 1, 24, 24, 128, 128, 119056, 119056, layout="bthd"), name="write_clip"),
        # three sequences of different length are moved out of a cache of narrow heads, an odd number of tokens
        dict(_case("read", 3, 12, 12, 64, 64, 2077, 2077, ragged=True), name="read_ragged"),
        # a short clip is read back for the entry points that take bf16
        dict(_case("read", 1, 24, 24, 128, 128, 20280, 20280, layout="bthd"), name="read_clip"),
        # decoding of 32 sequences, four query heads to a key/value head: which 64 of up to 512 blocks each token reads
        dict(_case("select", 32, 32, 8, 128, 64, 1, 32768, ragged=True, causal=True, group=1, keep=64, first=1, last=2), name="select_token"),
        # a new 45 x 80 frame against a clip in the cache, 90 % of the blocks left out, a list for every 128 tokens
        dict(_case("select", 1, 24, 24, 128, 128, 3600, 118800, group=128, keep=93, last=1, layout="bthd"), name="select_frame"),
        # the smallest call: three drafted tokens on a short cache
        dict(_case("attn", 1, 2, 2, 64, 64, 3, 1088, causal=True), name="attn_draft"),
        # decoding of 32 sequences of different length
        dict(_case("attn", 32, 32, 8, 128, 64, 1, 32768, ragged=True, causal=True), name="attn_token_batch"),
        # the same with 64 blocks a token
        dict(_case("attn", 32, 32, 8, 128, 64, 1, 32768, ragged=True, causal=True, group=1, keep=64, first=1, last=2), name="attn_token_lists"),
        # one query token against two long clips
        dict(_case("attn", 1, 24, 24, 128, 128, 1, 237600), name="attn_token_long"),
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
        kind = rng.choice(["write", "read", "select", "attn", "attn", "attn"])
        head_dim, block = rng.choice([(128, 128), (128, 64), (64, 128), (64, 64)])
        batch = _log_int(rng, 1, 48)
        heads_kv = rng.choice([1, 2, 3, 8, 12, 24])
        heads = heads_kv * (rng.choice([1, 1, 2, 4, 5, 8]) if kind in ("select", "attn") else 1)
        kv = _log_int(rng, 1, 240000)
        t = rng.choice([1, 1, rng.randint(1, 8), _log_int(rng, 1, 4000), _log_int(rng, 100, 4000)])
        if kind in ("write", "read"):
            t = rng.choice([t, kv])
        t = min(t, kv)
        case = _case(kind, batch, heads, heads_kv, head_dim, block, t, kv, ragged=batch > 1 and rng.random() < 0.6,
                     causal=kind in ("select", "attn") and rng.random() < 0.5, layout=rng.choice(["bhtd", "bthd"]))
        blocks = -(-kv // block)
        if kind == "select" or (kind == "attn" and rng.random() < 0.4):
            # few blocks or up to a third of them; groups of one token while there are few, of 16 to 128 for frames
            case.update(group=1 if t <= 8 else rng.choice([16, 50, 64, 128]), keep=rng.randint(1, max(1, blocks // rng.choice([3, 10, 20]))),
                        first=rng.choice([0, 1]), last=rng.choice([1, 2]))
        if blocks > 16384 or heads > 96 or batch * heads_kv * kv * head_dim > 24 * 237600 * 128 or batch * heads * t > 24 * 4000:
            continue
        if kind == "attn" and not case["group"] and batch * heads * t * kv > 24 * 1560 * 20280:
            continue
        if kind == "attn" and case["group"] and _lists_cost(case) > 24 * 29 * 93 * 128:
            continue
        if _cost(case) <= most[kind]:
            return case


def _lists_cost(case):
    return case["batch"] * case["heads_kv"] * -(-case["t"] // case["group"]) * _list_len(case) * case["block"]


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


def _visible(case, n, r, row):
    return n - r + row + 1 if case["causal"] else n


def work(case):
    lens, rows = _lengths(case)
    hk, h, d, B = case["heads_kv"], case["heads"], case["head_dim"], case["block"]
    byt = flops = 0.0
    for n, r in zip(lens, rows):
        if case["kind"] == "write":
            # new rows in, codes out; of the block that was begun before, the keys' codes for the mean; scales and means
            byt += hk * d * (r * 6 + (n - r) % B) + hk * (r / B + 1) * (16 + d)
            flops += 4.0 * hk * r * d
        elif case["kind"] == "read":
            byt += hk * d * r * 6
            flops += 2.0 * hk * r * d
        elif case["kind"] == "select":
            groups, blocks = -(-r // case["group"]), -(-n // B)
            byt += hk * blocks * (d + 4) + h * r * d * 2 + hk * groups * (_list_len(case) + 1) * 4
            flops += 2.0 * hk * groups * blocks * d
        else:
            keys = float(n)
            if case["group"]:
                keys = min(keys, float(_list_len(case)) * B)
                total = h * r * keys
                once = min(float(n), -(-r // case["group"]) * keys) * hk
            else:
                total = h * (r * keys - (r * (r - 1) / 2.0 if case["causal"] else 0.0))
                once = hk * keys
            byt += once * d * 2 + h * r * (d * 4 + 4)
            flops += 4.0 * total * d
    return {"bytes": byt, "flops": flops}


# ---- layout of a page, in torch ------------------------------------------------------------------
def _pack_k(x):
    """[..., B, d] -> [..., B*d]: 16 keys x 64 channels in one piece, in it runs of 16 channels of a key."""
    B, d = x.shape[-2:]
    n = x.dim() - 2
    x = x.reshape(*x.shape[:-2], B // 16, 16, d // 64, 4, 16)
    return x.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*x.shape[:n], B * d)


def _unpack_k(x, B, d):
    n = x.dim() - 1
    x = x.reshape(*x.shape[:-1], B // 16, d // 64, 4, 16, 16)
    return x.permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).reshape(*x.shape[:n], B, d)


def _pack_v(x):
    """[..., B, d] -> [..., B*d]: 64 keys x 16 channels in one piece, in it runs of 16 keys 16 t + 4 g + i (t, i) of a channel."""
    B, d = x.shape[-2:]
    n = x.dim() - 2
    x = x.reshape(*x.shape[:-2], B // 64, 4, 4, 4, d // 16, 16)                       # kg, t, g, i, tile, channel
    return x.permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3).reshape(*x.shape[:n], B * d)


def _unpack_v(x, B, d):
    n = x.dim() - 1
    x = x.reshape(*x.shape[:-1], B // 64, d // 16, 4, 16, 4, 4)                       # kg, tile, g, channel, t, i
    return x.permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3).reshape(*x.shape[:n], B, d)


def _exponent(amax, largest, least):
    """The least e >= `least` with amax <= largest * 2^e."""
    m, e = torch.frexp(amax)
    lm, le = math.frexp(largest)
    return torch.where(amax > 0, (e - le + (m > lm).to(e.dtype)), torch.full_like(e, least)).clamp(min=least)


def _finite(x):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x))


def _to_codes(x, e):
    """fp32 values over 2^e as e4m3; what is not finite becomes NaN."""
    y = torch.ldexp(x, -e)
    return torch.where(torch.isfinite(y), y, torch.full_like(y, math.nan)).to(E4M3)


def _mean_codes(k, n):
    """int8 codes and exponents of the mean of the first n rows of k [..., B, d] (zeros behind them)."""
    mean = _finite(k.to(F64)).sum(-2) / n.clamp(min=1).unsqueeze(-1)
    e = _exponent(mean.abs().amax(-1), 127.0, -100)
    return torch.round(torch.ldexp(mean, -e.unsqueeze(-1))).to(torch.int8), e


# ---- inputs --------------------------------------------------------------------------------------
def _smooth(gen, heads, tokens, d, noise, at=0):
    """Neighbouring tokens are alike, as those of a video are: four slow waves for each channel, and noise; [heads, tokens, d]."""
    f = torch.rand(heads, 4, 1, generator=gen, device="cuda") * 60 + 3
    pos = torch.arange(at, at + tokens, device="cuda", dtype=F32) / 120000.0
    amp = torch.randn(2, heads, 4, d, generator=gen, device="cuda") * 0.5
    x = (torch.randn(heads, tokens, d, generator=gen, device="cuda") * noise)
    theta = 2 * math.pi * f * pos
    x += torch.matmul(torch.sin(theta).transpose(1, 2), amp[0]) + torch.matmul(torch.cos(theta).transpose(1, 2), amp[1])
    return x


def _as_layout(x, layout):
    x = x.to(torch.bfloat16)
    return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if layout == "bthd" else x.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    b, h, hk, d, B, t = (case[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t"))
    lens, rows = _lengths(case)
    blocks = [-(-n // B) for n in lens]
    width = max(blocks)
    pages = sum(blocks) + 3
    table = torch.full((b, width), -1, dtype=torch.int32)
    # pages are handed out in no order; the last one never
    order = torch.randperm(pages - 1, generator=torch.Generator().manual_seed(int(seed) + 1))
    at = 0
    for i, n in enumerate(blocks):
        table[i, :n] = order[at:at + n].to(torch.int32)
        at += n
    s = {"case": case, "table": table.cuda(), "k_codes": torch.zeros(pages, hk, B * d, dtype=torch.uint8, device="cuda"),
         "v_codes": torch.zeros(pages, hk, B * d, dtype=torch.uint8, device="cuda"),
         "scales": torch.zeros(pages, hk, 4, dtype=F32, device="cuda"), "k_mean": torch.zeros(pages, hk, d, dtype=torch.int8, device="cuda")}
    for i, n in enumerate(lens):
        held = n - rows[i] if case["kind"] == "write" else n
        nb = -(-held // B)
        if nb == 0:
            continue
        page = table[i, :nb].cuda().long()
        left = (held - torch.arange(nb, device="cuda") * B).clamp(max=B)
        there = (torch.arange(B, device="cuda") < left[:, None])[:, None, :, None]
        for which in ("k", "v"):
            x = _smooth(gen, hk, nb * B, d, 0.5) if which == "k" else torch.randn(hk, nb * B, d, generator=gen, device="cuda")
            x = x.to(torch.bfloat16).to(F32).reshape(hk, nb, B, d).transpose(0, 1)
            x = torch.where(there, x, torch.zeros_like(x))
            e = _exponent(x.abs().amax((-1, -2)), 448.0, -126)
            c = _to_codes(x, e[..., None, None])
            pack = _pack_k if which == "k" else _pack_v
            s[which + "_codes"][page] = pack(c.view(torch.uint8))
            s["scales"][page, :, 0 if which == "k" else 1] = torch.ldexp(torch.ones_like(e, dtype=F32), e)
            if which == "k":
                code, em = _mean_codes(torch.ldexp(c.to(F32), e[..., None, None]), left[:, None].expand(nb, hk))
                s["k_mean"][page] = code
                s["scales"][page, :, 2] = torch.ldexp(torch.ones_like(em, dtype=F32), em)
            del x, c
    i32 = dict(dtype=torch.int32, device="cuda")
    s["kv_len"], s["q_len"] = torch.tensor(lens, **i32), torch.tensor(rows, **i32)
    s["start"] = s["kv_len"] - s["q_len"]
    if case["kind"] in ("write", "read"):
        shape = (b, hk, t, d)
        if case["kind"] == "write":
            s["K"] = _as_layout(torch.stack([_smooth(gen, hk, t, d, 0.5) for _ in range(b)]), case["layout"])
            s["V"] = _as_layout(torch.randn(shape, generator=gen, device="cuda"), case["layout"])
        else:
            s["K"], s["V"] = (_as_layout(torch.zeros(shape, device="cuda"), case["layout"]) for _ in range(2))
        return s
    s["Q"] = _as_layout(torch.stack([_smooth(gen, h, t, d, 0.5) for _ in range(b)]), case["layout"])
    if case["group"]:
        groups = -(-t // case["group"])
        s["block_idx"] = torch.full((b, hk, groups, _list_len(case)), -1, **i32)
        s["kept"] = torch.zeros(b, hk, groups, **i32)
        if case["kind"] == "attn":                    # the lists are an input here
            s["block_idx"], s["kept"] = _select(s)
    if case["kind"] == "attn":
        s["O"] = torch.zeros_like(s["Q"])
        s["lse"] = torch.zeros(b, h, t, dtype=F32, device="cuda")
    return s


# ---- the plain forms -----------------------------------------------------------------------------
def _write(s):
    c = s["case"]
    b, hk, d, B, t = (c[k] for k in ("batch", "heads_kv", "head_dim", "block", "t"))
    J = min((t - 1) // B + 2, s["table"].shape[1])
    start, count = s["start"].long(), s["q_len"].long()
    j0 = (start // B).clamp(max=s["table"].shape[1] - J)
    blk = j0[:, None] + torch.arange(J, device="cuda")                                   # [b, J]
    page = torch.gather(s["table"].long(), 1, blk)
    pos = blk[..., None] * B + torch.arange(B, device="cuda")                            # [b, J, B]
    new = (pos >= start[:, None, None]) & (pos < (start + count)[:, None, None])
    old = pos < start[:, None, None]
    touched = new.any(-1) & (page >= 0)
    kept_before = old.any(-1) & touched
    safe = torch.where(page >= 0, page, torch.full_like(page, s["k_codes"].shape[0] - 1))
    row = (pos - start[:, None, None]).clamp(0, t - 1).reshape(b, 1, J * B, 1).expand(b, hk, J * B, d)
    own_new, own_old = new[:, :, None, :, None], old[:, :, None, :, None]                # [b, J, 1, B, 1]
    there = touched[:, :, None]
    for which, X, pack, unpack, col in (("k", s["K"], _pack_k, _unpack_k, 0), ("v", s["V"], _pack_v, _unpack_v, 1)):
        x = torch.gather(X, 2, row).reshape(b, hk, J, B, d).transpose(1, 2).to(F32)      # [b, J, hk, B, d]
        x = torch.where(own_new, x, torch.zeros_like(x))
        e = _exponent(_finite(x).abs().amax((-1, -2)), 448.0, -126)
        was = s[which + "_codes"][safe]
        held = s["scales"][safe][..., col]
        e = torch.where(kept_before[:, :, None], torch.maximum(e, torch.frexp(held)[1] - 1), e)
        before = unpack(was, B, d).view(E4M3).to(F32) * held[..., None, None]
        x = torch.where(own_old & kept_before[:, :, None, None, None], before, x)
        code = _to_codes(x, e[..., None, None])
        s[which + "_codes"][safe] = torch.where(there[..., None], pack(code.view(torch.uint8)), was)
        s["scales"][..., col][safe] = torch.where(there, torch.ldexp(torch.ones_like(held), e), held)
        if which == "k":
            n = (old | new).sum(-1)[:, :, None].expand(b, J, hk)
            mean, em = _mean_codes(torch.ldexp(code.to(F32), e[..., None, None]), n)
            s["k_mean"][safe] = torch.where(there[..., None], mean, s["k_mean"][safe])
            s["scales"][..., 2][safe] = torch.where(there, torch.ldexp(torch.ones_like(held), em), s["scales"][..., 2][safe])


def _rows_of(s, codes, col, page, unpack):
    """The values of pages [...] as fp32 [..., hk, B, d] (0 where there is no page)."""
    c = s["case"]
    safe = page.clamp(min=0)
    x = unpack(codes[safe], c["block"], c["head_dim"]).view(E4M3).to(F32) * s["scales"][safe][..., col][..., None, None]
    return torch.where((page >= 0)[..., None, None, None], x, torch.zeros_like(x))


def _read(s):
    c = s["case"]
    b, hk, d, B, t = (c[k] for k in ("batch", "heads_kv", "head_dim", "block", "t"))
    pos = s["start"].long()[:, None] + torch.arange(t, device="cuda")
    there = (torch.arange(t, device="cuda") < s["q_len"].long()[:, None])[:, None, :, None]
    page = s["table"].long()
    at = pos.clamp(max=page.shape[1] * B - 1)[:, None, :, None].expand(b, hk, t, d)
    for codes, col, unpack, X in ((s["k_codes"], 0, _unpack_k, s["K"]), (s["v_codes"], 1, _unpack_v, s["V"])):
        x = _rows_of(s, codes, col, page, unpack).transpose(1, 2).reshape(b, hk, -1, d)
        X.copy_(torch.where(there, torch.gather(x, 2, at).to(torch.bfloat16), X))


def _group_rows(x, group):
    """[b, h, t, ...] -> [b, h, groups, group, ...], zeros behind."""
    t = x.shape[2]
    groups = -(-t // group)
    full = torch.zeros(*x.shape[:2], groups * group, *x.shape[3:], dtype=x.dtype, device=x.device)
    full[:, :, :t] = x
    return full.reshape(*x.shape[:2], groups, group, *x.shape[3:])


def _select(s):
    c = s["case"]
    b, h, hk, d, B, t, group = (c[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t", "group"))
    groups, L, M = -(-t // group), _list_len(c), s["table"].shape[1]
    kv, r = s["kv_len"].long(), s["q_len"].long()
    q = torch.where((torch.arange(t, device="cuda") < r[:, None])[:, None, :, None], _finite(s["Q"].to(F64)), 0.0)
    q = _group_rows(q, group).reshape(b, hk, h // hk, groups, group, d).sum((2, 4))       # [b, hk, groups, d]
    e = _exponent(q.abs().amax(-1), 127.0, -100)
    q = torch.round(torch.ldexp(q, -e.unsqueeze(-1)))
    safe = s["table"].long().clamp(min=0)
    mean = s["k_mean"][safe].transpose(1, 2).to(F64)                                      # [b, hk, M, d]
    score = torch.matmul(q, mean.transpose(-1, -2).contiguous()) * s["scales"][safe][..., 2].transpose(1, 2)[:, :, None, :].to(F64)
    lo = torch.arange(groups, device="cuda") * group
    first = (kv - r)[:, None] + lo                                                        # [b, groups] first and last position
    last = (kv - r)[:, None] + torch.minimum(lo + group, r[:, None]) - 1
    some = lo < r[:, None]
    blk = torch.arange(M, device="cuda")
    seen = torch.where(torch.full_like(last, c["causal"], dtype=torch.bool), last // B + 1, ((kv + B - 1) // B)[:, None])
    visible = (blk < seen[..., None]) & some[..., None] & (s["table"].long() >= 0)[:, None, :]
    forced = (blk < c["first"]) | ((blk > (first // B)[..., None] - c["last"]) & (blk <= (last // B)[..., None]) & (c["last"] > 0))
    score = torch.where(forced[:, None], torch.full_like(score, math.inf), score)
    score = torch.where(visible[:, None], score, torch.full_like(score, -math.inf))
    place = torch.argsort(torch.argsort(score, dim=-1, descending=True, stable=True), dim=-1, stable=True)
    keep = (visible & forced).sum(-1).clamp(min=c["keep"])[:, None, :, None]
    kept = (place < keep) & visible[:, None]
    idx = torch.where(kept, blk.expand_as(kept), torch.full_like(blk, M).expand_as(kept)).sort(-1).values[..., :L]
    return torch.where(idx < M, idx, torch.full_like(idx, -1)).to(torch.int32), kept.sum(-1).to(torch.int32)


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
    q = _group_rows(s["Q"].to(F32), per).reshape(b, hk, h // hk, groups, per, d).transpose(2, 3)      # [b, hk, groups, G, per, d]
    q = q.reshape(b, hk, groups, h // hk * per, d)
    if group:
        blk = s["block_idx"].long()                                                       # [b, hk, groups, L]
        page = torch.where(blk >= 0, torch.gather(s["table"].long()[:, None, None].expand(b, hk, groups, -1), 3, blk.clamp(min=0)), -1)
        head = torch.arange(hk, device="cuda")[None, :, None, None].expand_as(page)
        safe = page.clamp(min=0)
        k = _unpack_k(s["k_codes"][safe, head], B, d).view(E4M3).to(F32) * s["scales"][safe, head, 0][..., None, None]
        v = _unpack_v(s["v_codes"][safe, head], B, d).view(E4M3).to(F32) * s["scales"][safe, head, 1][..., None, None]
        k, v = k.reshape(b, hk, groups, -1, d), v.reshape(b, hk, groups, -1, d)
    else:
        page = s["table"].long()
        blk = torch.arange(page.shape[1], device="cuda").expand(b, 1, 1, -1)
        k = _rows_of(s, s["k_codes"], 0, page, _unpack_k).transpose(1, 2).reshape(b, hk, 1, -1, d)
        v = _rows_of(s, s["v_codes"], 1, page, _unpack_v).transpose(1, 2).reshape(b, hk, 1, -1, d)
        page = page[:, None, None]
    key = (blk[..., None] * B + torch.arange(B, device="cuda")).flatten(-2)               # [b, hk|1, groups|1, n]
    there = (page >= 0)[..., None].expand(*page.shape, B).flatten(-2) & (key >= 0)
    kv, r = s["kv_len"].long(), s["q_len"].long()
    row = torch.arange(groups * per, device="cuda").reshape(groups, per).repeat(1, h // hk)            # [groups, G * per]
    bound = (kv - r)[:, None, None] + row + 1 if c["causal"] else kv[:, None, None].expand(b, *row.shape)
    seen = there[..., None, :] & (key[..., None, :] < torch.minimum(bound, kv[:, None, None])[:, None, :, :, None])
    o, lse = _softmax_rows(q, k, v, seen)
    back = lambda x: x.reshape(b, hk, groups, h // hk, per, *x.shape[4:]).transpose(2, 3).reshape(b, h, groups * per, *x.shape[4:])[:, :, :t]
    mine = (torch.arange(t, device="cuda") < r[:, None])[:, None]
    s["O"].copy_(torch.where(mine[..., None], back(o).to(torch.bfloat16), s["O"]))
    s["lse"].copy_(torch.where(mine, back(lse), s["lse"]))


# ---- one pass ------------------------------------------------------------------------------------
def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "write":
        return {"k": s["k_codes"].view(E4M3), "v": s["v_codes"].view(E4M3), "scales": s["scales"], "mean": s["k_mean"]}
    if kind == "read":
        return {"k": s["K"], "v": s["V"]}
    if kind == "select":
        return {"block_idx": s["block_idx"], "kept": s["kept"]}
    return {"o": s["O"], "lse": s["lse"]}


def _run_own(s):
    from paper_2511_19835_amd import binding as rb
    c = s["case"]
    if "cache" not in s:                              # the records that a program makes once for its cache and its tensors
        s["cache"] = rb.cache_of(s["k_codes"], s["v_codes"], s["scales"], s["k_mean"], s["table"], c["block"])
        s["rows"] = rb.make_rows(s["K"] if "K" in s else s["Q"])
        select, attn = rb.rsa_cache_workspace_bytes(s["cache"], s["rows"], c["group"])
        s["ws"] = torch.empty(max(256, select if c["kind"] == "select" else attn), dtype=torch.uint8, device="cuda")
        s["flags"] = rb.RSA_CACHE_CAUSAL if c["causal"] else 0
    if c["kind"] == "write":
        rb.rsa_cache_write(s["cache"], s["rows"], s["K"], s["V"], s["start"], s["q_len"])
    elif c["kind"] == "read":
        rb.rsa_cache_read(s["cache"], s["rows"], s["start"], s["q_len"], s["K"], s["V"])
    elif c["kind"] == "select":
        rb.rsa_cache_select(s["cache"], s["rows"], s["Q"], s["kv_len"], s["q_len"], c["group"], c["keep"], c["first"], c["last"],
                            s["flags"], s["block_idx"], s["kept"], s["ws"])
    else:
        rb.rsa_cache_attn(s["cache"], s["rows"], s["Q"], s["kv_len"], s["q_len"], 0.0, s["flags"], s.get("block_idx"), s.get("kept"),
                          c["group"], s["O"], s["lse"], s["ws"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        _run_own(s)
    elif kind == "write":
        _write(s)
    elif kind == "read":
        _read(s)
    elif kind == "select":
        s["block_idx"], s["kept"] = _select(s)
    else:
        _attn(s)
    return _outputs(s)


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _value64(codes):
    """e4m3 bytes as fp64, from their bits: (-1)^s (1 + m/8) 2^(x-7), m/8 2^-6 at x = 0, NaN at 127."""
    u = codes.to(torch.int32)
    x, m = (u >> 3) & 15, (u & 7).to(F64)
    v = torch.where(x == 0, m * 2.0 ** -9, (8 + m) * torch.exp2((x - 10).to(F64)))
    v = torch.where((u & 127) == 127, torch.full_like(v, math.nan), v)
    return torch.where(u >= 128, -v, v)


def _round64(x):
    """fp64 to the nearest value of e4m3 (even on ties), |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3)
    return torch.round(x / step) * step


def _index_k(B, d):
    """Place of (token, channel) among the codes of a page's keys."""
    t, ch = torch.arange(B, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    return ((t // 16 * (d // 64) + ch // 64) * 4 + ch % 64 // 16) * 256 + t % 16 * 16 + ch % 16


def _index_v(B, d):
    t, ch = torch.arange(B, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    return ((t // 64 * (d // 16) + ch // 16) * 4 + t % 16 // 4) * 256 + ch % 16 * 16 + t % 64 // 16 * 4 + t % 4


def _tokens64(s, i, j, lo, hi):
    """Keys and values of tokens lo..hi-1 of head j, sequence i, fp64 [hi - lo, d]."""
    c = s["case"]
    B, d = c["block"], c["head_dim"]
    tok = torch.arange(lo, hi, device="cuda")
    page = s["table"][i].long()[tok // B]
    out = []
    for name, col, index in (("k_codes", 0, _index_k(B, d)), ("v_codes", 1, _index_v(B, d))):
        flat = page[:, None] * (c["heads_kv"] * B * d) + j * B * d + index[tok % B]
        out.append(_value64(s[name].reshape(-1)[flat]) * s["scales"][page, j, col].to(F64)[:, None])
    return out


def _least(amax, largest, least):
    """The least e >= `least` with amax <= largest * 2^e, for one number."""
    if amax == 0:
        return least
    e = math.floor(math.log2(amax / largest)) - 1
    while amax > math.ldexp(largest, e):
        e += 1
    return max(e, least)


def _exact_write(s):
    c = s["case"]
    hk, d, B = c["heads_kv"], c["head_dim"], c["block"]
    lens, rows = _lengths(c)
    if sum(rows) * hk > 200000:
        return None
    k, v = _value64(s["k_codes"]), _value64(s["v_codes"])
    scales, mean = s["scales"].to(F64), s["k_mean"].clone()
    for i, (n, r) in enumerate(zip(lens, rows)):
        for blk in range((n - r) // B, -(-n // B)):
            lo, hi, page = max(n - r, blk * B), min(n, blk * B + B), int(s["table"][i, blk])
            for j in range(hk):
                for vals, X, col, index in ((k, s["K"], 0, _index_k(B, d)), (v, s["V"], 1, _index_v(B, d))):
                    new = X[i, j, lo - (n - r):hi - (n - r)].to(F64)
                    e = _least(float(new.abs().max()), 448.0, -126)
                    block = torch.zeros(B, d, dtype=F64, device="cuda")
                    if lo > blk * B:
                        was = float(scales[page, j, col])
                        e = max(e, round(math.log2(was)))
                        block[:lo - blk * B] = vals[page, j][index[:lo - blk * B]] * was
                    block[lo - blk * B:hi - blk * B] = new
                    block = _round64(block / 2.0 ** e)
                    vals[page, j][index] = block
                    scales[page, j, col] = 2.0 ** e
                    if col == 0:
                        m = block.sum(0) * 2.0 ** e / (hi - blk * B)
                        e = _least(float(m.abs().max()), 127.0, -100)
                        mean[page, j] = torch.round(m / 2.0 ** e).to(torch.int8)
                        scales[page, j, 2] = 2.0 ** e
    return {"k": k, "v": v, "scales": scales, "mean": mean}


def _exact_read(s):
    c = s["case"]
    lens, rows = _lengths(c)
    K, V = (torch.zeros(c["batch"], c["heads_kv"], c["t"], c["head_dim"], dtype=F64, device="cuda") for _ in range(2))
    for i, (n, r) in enumerate(zip(lens, rows)):
        for j in range(c["heads_kv"]):
            K[i, j, :r], V[i, j, :r] = _tokens64(s, i, j, n - r, n)
    return {"k": K, "v": V}


def _exact_select(s):
    c = s["case"]
    b, h, hk, d, B, t, group = (c[k] for k in ("batch", "heads", "heads_kv", "head_dim", "block", "t", "group"))
    lens, rows = _lengths(c)
    groups, G = -(-t // group), h // hk
    if b * hk * groups > 3000:
        return None
    idx = torch.full((b, hk, groups, _list_len(c)), -1, dtype=torch.int32)
    kept = torch.zeros(b, hk, groups, dtype=torch.int32)
    for i, (n, r) in enumerate(zip(lens, rows)):
        page = s["table"][i].long()[:-(-n // B)]
        for j in range(hk):
            mean, scale = s["k_mean"][page, j].to(F64), s["scales"][page, j, 2].to(F64)
            for g in range(-(-r // group)):
                hi = min(r, g * group + group)
                q = s["Q"][i, j * G:j * G + G, g * group:hi].to(F64).sum((0, 1))
                q = torch.round(q / 2.0 ** _least(float(q.abs().max()), 127.0, -100))
                score = ((mean * q).sum(1) * scale).tolist()
                p0, p1 = n - r + g * group, n - r + hi - 1
                seen = p1 // B + 1 if c["causal"] else -(-n // B)
                must = {m for m in range(seen) if m < c["first"] or (c["last"] and p0 // B - c["last"] < m <= p1 // B)}
                rest = sorted((m for m in range(seen) if m not in must), key=lambda m: (-score[m], m))
                row = sorted(must | set(rest[:max(0, c["keep"] - len(must))]))
                idx[i, j, g, :len(row)] = torch.tensor(row, dtype=torch.int32)
                kept[i, j, g] = len(row)
    return {"block_idx": idx, "kept": kept}


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
    return {"write": _exact_write, "read": _exact_read, "select": _exact_select, "attn": _exact_attn}[case["kind"]](s)
