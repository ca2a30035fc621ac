"""Performance cases of the language-model operators: the attention block of a quantised decoder.

Three groups, each reached through the binding's calls where `own` is true:

* append: q and k rotated by their positions, k and v quantised to 4 bits a value and written into a
  paged cache (ifq_kv4_append), and the written tokens read back as the values they stand for (ifq_kv4_read);
* attention: queries against the 4-bit paged cache (ifq_kv4_attention): one token a sequence, a few
  tokens, and chunks of a prompt, with an optional sliding window whose first tokens stay visible;
* fp8: a product in e4m3 with a float scale for each block of 128 (ifq_fp8_quantize on the activations,
  ifq_fp8_matmul with weights that were quantised once).

Where `own` is false run() computes the same in elementary torch operations in 32 bits.

The cache's format.  A page holds page_size tokens; the cache is [pages][kv_heads][page_size / 16] groups
of 16 tokens, each group 16 * D + 128 bytes for head size D: the K codes (8 * D bytes), the V codes
(8 * D bytes), 16 (scale, min) pairs of float16 for K and 16 for V.  A value is code * scale + min.  Codes
are 4-bit fields, the lower-numbered one in the low half of its byte.  With DB = min(D, 128), K codes are
[D / DB][16 tokens][DB]; V codes are [D / DB][2][8][4][DB / 32][2][4] with token = 8 * (second axis) +
2 * (fourth) + (sixth) and dimension = DB / 8 * (third) + 4 * (fifth) + (seventh): two neighbouring tokens'
codes of the same four dimensions share a 32-bit word.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 16


# ------------------------------------------------------------------------------------ cases


def _append(name, tokens, hq, hk, d, dtype, rope="halves", rot=None, page=64):
    return {"name": name, "do": "append", "tokens": tokens, "hq": hq, "hk": hk, "d": d, "dtype": dtype, "rope": rope,
            "rot": d if rot is None else rot, "page": page, "history": 4096}


def _attn(name, seqs, nq, lo, hi, hq, hk, d, dtype, page=64, window=0, sinks=0):
    return {"name": name, "do": "attention", "seqs": seqs, "nq": nq, "len_lo": lo, "len_hi": hi, "hq": hq, "hk": hk,
            "d": d, "dtype": dtype, "page": page, "window": window, "sinks": sinks}


def _fp8(name, m, n, k, dtype="bf16", out="bf16"):
    return {"name": name, "do": "fp8", "m": m, "n": n, "k": k, "dtype": dtype, "out": out}


def listed():
    return [
        # one new token of one conversation: a latency-bound call
        _append("append_1_token", 1, 32, 8, 128, "bf16"),
        # a batch of odd size with small heads, a quarter of each rotated in neighbouring pairs
        _append("append_777_d64_pairs", 777, 16, 2, 64, "f16", "pairs", 16, 16),
        # the prompt of a long request, in one call
        _append("append_8191_prompt", 8191, 32, 8, 128, "bf16"),
        # one token of one short conversation: a latency-bound call
        _attn("decode_1x517", 1, 1, 517, 517, 32, 8, 128, "bf16", 16),
        # a serving batch of conversations of every length
        _attn("decode_48_ragged_8192", 48, 1, 1, 8192, 32, 8, 128, "bf16"),
        # one token over a long document: few rows, the keys are what is split
        _attn("decode_1x131072", 1, 1, 131072, 131072, 32, 8, 128, "bf16"),
        # a batch of long streams that see their last 1024 tokens and the first four
        _attn("decode_64_window1024_sinks4", 64, 1, 1500, 16384, 16, 2, 64, "f16", 16, 1024, 4),
        # a few drafted tokens a sequence, to be verified in one call
        _attn("verify_16x5_4096", 16, 5, 257, 4096, 64, 8, 128, "f16", 32),
        # chunks of two prompts over what their caches already hold
        _attn("chunk_2x2048_8192", 2, 2048, 2100, 8192, 32, 8, 128, "bf16", 128),
        # one token through a large projection: the weights are what is read
        _fp8("fp8_1x4096x9216", 1, 4096, 9216),
        # a small odd batch, with a last block that is not full
        _fp8("fp8_37x6152x4112", 37, 6152, 4112, "f16", "f16"),
        # a prompt through the same projection
        _fp8("fp8_4096x4096x9216", 4096, 4096, 9216),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v if v <= 1024 else min(v | 1, hi)  # the large ones odd


# query heads, key heads, head size
HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (16, 2, 64), (16, 16, 128), (28, 4, 128), (8, 1, 256), (16, 8, 256),
         (12, 4, 64)]


def draw(rng):
    most = {"append": 3e8, "attention": 4e9, "fp8": 6e9}
    while True:
        do = rng.choice(["append", "attention", "attention", "attention", "fp8", "fp8"])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        if do == "append":
            hq, hk, d = rng.choice(HEADS)
            c = _append("", _log(rng, 1, 8191), hq, hk, d, dtype, rng.choice(["halves", "halves", "pairs"]),
                        rng.choice([d, d, d // 2]), rng.choice([16, 32, 64, 128]))
        elif do == "attention":
            hq, hk, d = rng.choice(HEADS)
            kind = rng.choice(["decode", "decode", "decode", "few", "chunk"])
            if kind == "chunk":
                seqs, nq, hi = _log(rng, 1, 8), _log(rng, 33, 2048), _log(rng, 64, 8192)
            else:
                seqs, nq, hi = _log(rng, 1, 128), 1 if kind == "decode" else rng.randint(2, 16), _log(rng, 1, 131072)
            hi = max(hi, nq)
            window = _log(rng, 32, 4096) if rng.random() < 0.3 else 0
            c = _attn("", seqs, nq, hi if rng.random() < 0.3 else min(nq, hi), hi, hq, hk, d, dtype,
                      rng.choice([16, 32, 64, 128]), window, rng.choice([0, 1, 4, 20]) if window else 0)
            # the plain form's own arrays: values of the padded cache, and scores
            if max(seqs * hi * hk * d, seqs * nq * hi * hq) > 4e8:
                continue
        else:
            n = rng.choice([128 * 2 ** rng.randint(2, 6), 8 * _log(rng, 16, 1024) + 1])
            k = rng.choice([128 * 2 ** rng.randint(2, 6), 16 * (2 * _log(rng, 4, 256) + 1)])
            c = _fp8("", _log(rng, 1, 4096), n, k, dtype, rng.choice([dtype, dtype, "f32"]))
        del c["name"]
        w = work(c)
        if max(w["bytes"], w["flops"] / 50) <= most[do]:
            return c


# ------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(8076 + seed)
    return g


def _quantise4(x):
    """float32 [..., D] -> codes uint8 [..., D] and (scale, min) float16 [..., 2]: the cache's definition, in IEEE
    float32 and in this order."""
    x = x.clamp(-65504.0, 65504.0)
    lo = x.amin(-1, keepdim=True)
    sc = ((x.amax(-1, keepdim=True) - lo) / 15.0).half()
    lo = lo.half()
    s, m = sc.to(x.dtype), lo.to(x.dtype)
    code = torch.round((x - m) / s).clamp(0.0, 15.0)
    code = torch.where((s == 0) | torch.isnan(s), torch.zeros_like(code), code)
    return code.to(torch.uint8), torch.cat([sc, lo], -1)


def _k_axes(d):
    db = min(d, 128)
    return d // db, db


def _pack_k(codes):
    """uint8 codes [..., 16, D] -> bytes [..., 8 * D]"""
    nb, db = _k_axes(codes.shape[-1])
    lead = codes.shape[:-2]
    c = codes.view(*lead, 16, nb, db // 2, 2)
    return (c[..., 0] | (c[..., 1] << 4)).transpose(-3, -2).reshape(*lead, -1)


def _unpack_k(b, d):
    nb, db = _k_axes(d)
    lead = b.shape[:-1]
    c = b.view(*lead, nb, 16, db // 2).transpose(-3, -2)
    return torch.stack([c & 15, c >> 4], -1).reshape(*lead, 16, d)


def _pack_v(codes):
    nb, db = _k_axes(codes.shape[-1])
    lead, n = codes.shape[:-2], codes.dim() - 2
    # token (half, pair, odd), dimension (block, slice, word, byte, nibble)
    c = codes.view(*lead, 2, 4, 2, nb, 8, db // 32, 2, 2)
    c = c[..., 0] | (c[..., 1] << 4)
    order = [n + i for i in (3, 0, 4, 1, 5, 2, 6)]
    return c.permute(*range(n), *order).reshape(*lead, -1)


def _unpack_v(b, d):
    nb, db = _k_axes(d)
    lead, n = b.shape[:-1], b.dim() - 1
    c = b.view(*lead, nb, 2, 8, 4, db // 32, 2, 2)
    order = [n + i for i in (1, 3, 5, 0, 2, 4, 6)]
    c = c.permute(*range(n), *order)
    return torch.stack([c & 15, c >> 4], -1).reshape(*lead, 16, d)


def _pack_groups(kc, kp, vc, vp):
    """codes [..., 16, D] and parameters float16 [..., 16, 2] of whole groups -> bytes [..., 16 * D + 128]"""
    flat = lambda p: p.contiguous().view(torch.uint8).reshape(*p.shape[:-2], 64)  # noqa: E731
    return torch.cat([_pack_k(kc), _pack_v(vc), flat(kp), flat(vp)], -1)


def _unpack_groups(b, d):
    """bytes [..., 16 * D + 128] -> codes and float16 parameters (k, v)"""
    kb, vb, kp, vp = b.split([8 * d, 8 * d, 64, 64], -1)
    par = lambda p: p.contiguous().view(torch.float16).reshape(*p.shape[:-1], 16, 2)  # noqa: E731
    return _unpack_k(kb.contiguous(), d), par(kp), _unpack_v(vb.contiguous(), d), par(vp)


def _values(codes, par, dtype=torch.float32):
    return codes.to(dtype) * par[..., :1].to(dtype) + par[..., 1:].to(dtype)


def _keys_and_values(g, shape, d):
    """Keys with a few channels that sit off zero, as rotated keys do, and values without."""
    off = torch.randn(d, generator=g, device=DEV) * 0.5
    k = torch.randn(*shape, d, generator=g, device=DEV) + off
    v = torch.randn(*shape, d, generator=g, device=DEV) * 0.5
    return k, v


def _filled_cache(g, pages, hk, page, d):
    """A cache whose every slot holds a token's quantised keys and values."""
    cache = torch.empty(pages, hk, page // GROUP, 16 * d + 128, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (hk * page * d))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k, v = _keys_and_values(g, (n, hk, page // GROUP, GROUP), d)
        cache[p:p + n] = _pack_groups(*_quantise4(k), *_quantise4(v))
    return cache


def _prepare_append(c, g):
    t, hq, hk, d, page = c["tokens"], c["hq"], c["hk"], c["d"], c["page"]
    dt = TYPES[c["dtype"]]
    # q, k and v of a token side by side, as a fused projection leaves them
    qkv = torch.randn(t, (hq + 2 * hk) * d, generator=g, device=DEV).to(dt)
    # a prompt takes the positions in order; a batch of decoding sequences sits anywhere
    if t > 1024:
        pos = torch.arange(t, device=DEV, dtype=torch.int32)
        slots = torch.arange(t, device=DEV, dtype=torch.int64)
        pages = -(-t // page)
        slots = torch.randperm(pages, generator=g, device=DEV)[slots // page] * page + slots % page
    else:
        pages = max(t, 8)
        pos = torch.randint(0, c["history"], (t,), generator=g, device=DEV, dtype=torch.int32)
        slots = torch.randperm(pages, generator=g, device=DEV)[:t] * page + pos % page
    rows = max(c["history"], t)
    inv = 10000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"])
    ang = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * inv
    return {"qkv": qkv, "q": qkv[:, :hq * d], "k": qkv[:, hq * d:(hq + hk) * d], "v": qkv[:, (hq + hk) * d:],
            "cos": ang.cos().float().contiguous(), "sin": ang.sin().float().contiguous(), "pos": pos, "slots": slots,
            "cache": torch.zeros(pages, hk, page // GROUP, 16 * d + 128, dtype=torch.uint8, device=DEV),
            "q_out": torch.empty(t, hq * d, dtype=dt, device=DEV),
            "k_out": torch.empty(t, hk * d, dtype=dt, device=DEV),
            "v_out": torch.empty(t, hk * d, dtype=dt, device=DEV)}


def _lengths(c, g):
    """Tokens in each sequence's cache, and how many of its last ones ask."""
    n = c["seqs"]
    lens = torch.randint(c["len_lo"], c["len_hi"] + 1, (n,), generator=g, device=DEV)
    # not every sequence brings as many; len_lo is at least nq
    nq = c["nq"] - torch.arange(n, device=DEV) * 5 % (c["nq"] // 2 + 1)
    return lens, nq


def _prepare_attention(c, g):
    n, hq, hk, d, page = c["seqs"], c["hq"], c["hk"], c["d"], c["page"]
    dt = TYPES[c["dtype"]]
    lens, nq = _lengths(c, g)
    starts = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    starts[1:] = nq.cumsum(0)
    row = -(-c["len_hi"] // page)
    need = (lens + page - 1) // page
    first = torch.cumsum(need, 0) - need
    pages = int(need.sum()) + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = (first[:, None] + torch.arange(row, device=DEV)).clamp_max(pages - 1)
    table = torch.where(torch.arange(row, device=DEV) < need[:, None], perm[at], torch.zeros_like(perm[at]))
    total = int(starts[-1])
    q = (torch.randn(total, hq * d, generator=g, device=DEV) * 1.5).to(dt)
    return {"q": q, "cache": _filled_cache(g, pages, hk, page, d), "table": table.contiguous(),
            "lens": lens.to(torch.int32), "starts": starts, "max_q": int(nq.max()), "max_len": int(lens.max()),
            "out": torch.empty_like(q), "lse": torch.empty(total, hq, device=DEV)}


def _prepare_fp8(c, g):
    m, n, k = c["m"], c["n"], c["k"]
    x = torch.randn(m, k, generator=g, device=DEV)
    x = (x * (1 + 8 * (torch.rand(k, generator=g, device=DEV) < 0.01))).to(TYPES[c["dtype"]])  # a few loud channels
    kb, nb = -(-k // 128), -(-n // 128)
    w = torch.zeros(nb * 128, kb * 128, device=DEV)
    w[:n, :k] = torch.randn(n, k, generator=g, device=DEV) * 0.02
    blocks = w.view(nb, 128, kb, 128)
    sw = (blocks.abs().amax((1, 3)) / 448.0).contiguous()
    wq = (blocks / sw[:, None, :, None]).view(nb * 128, kb * 128)[:n, :k].contiguous().to(torch.float8_e4m3fn)
    return {"x": x, "w": wq, "sw": sw, "xq": torch.empty(m, k, dtype=torch.float8_e4m3fn, device=DEV),
            "sx": torch.empty(kb, m, device=DEV), "out": torch.empty(m, n, dtype=TYPES[c["out"]], device=DEV)}


PREPARE = {"append": _prepare_append, "attention": _prepare_attention, "fp8": _prepare_fp8}


def prepare(case, seed):
    s = PREPARE[case["do"]](case, _gen(seed))
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------ the plain forms


def _rotate(x, cos, sin, rope, rot):
    """x [T, H, D]; cos, sin [T, rot / 2]"""
    cos, sin = cos[:, None], sin[:, None]
    if rope == "halves":
        a, b, rest = x.split([rot // 2, rot // 2, x.shape[-1] - rot], -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    y, rest = x.split([rot, x.shape[-1] - rot], -1)
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _code_offsets(d, device):
    """Where in a group the bytes of each token's codes are: [16, D / 2] for K and for V"""
    ids = torch.arange(8 * d, device=device)
    nb, db = _k_axes(d)
    k = ids.view(nb, 16, db // 2).transpose(0, 1).reshape(16, d // 2)
    v = ids.view(nb, 2, 8, 4, db // 32, 2, 2).permute(1, 3, 5, 0, 2, 4, 6).reshape(16, d // 2)
    return k, 8 * d + v


def _plain_append(s):
    c = s["case"]
    t, hq, hk, d, page = c["tokens"], c["hq"], c["hk"], c["d"], c["page"]
    dt = s["q"].dtype
    cos, sin = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
    q = _rotate(s["q"].float().reshape(t, hq, d), cos, sin, c["rope"], c["rot"])
    k = _rotate(s["k"].float().reshape(t, hk, d), cos, sin, c["rope"], c["rot"])
    kc, kp = _quantise4(k)
    vc, vp = _quantise4(s["v"].float().reshape(t, hk, d))
    # the bytes' places: page, head, group, token in the group
    slot, size = s["slots"], 16 * d + 128
    group = ((slot // page)[:, None] * hk + torch.arange(hk, device=DEV)) * (page // GROUP) + (slot % page // GROUP)[:, None]
    base, row = (group * size)[..., None], slot % GROUP
    ko, vo = _code_offsets(d, slot.device)
    ka, va = base + ko[row][:, None], base + vo[row][:, None]
    pa = base + (16 * d + 4 * row)[:, None, None] + torch.arange(4, device=DEV)
    flat = s["cache"].view(-1)
    pair = lambda x: x[..., 0::2] | (x[..., 1::2] << 4)  # noqa: E731
    flat[ka], flat[va] = pair(kc), pair(vc)
    flat[pa], flat[pa + 64] = kp.contiguous().view(torch.uint8), vp.contiguous().view(torch.uint8)
    # and read back
    split = lambda b: torch.stack([b & 15, b >> 4], -1).flatten(-2)  # noqa: E731
    kv = _values(split(flat[ka]), flat[pa].view(torch.float16))
    vv = _values(split(flat[va]), flat[pa + 64].view(torch.float16))
    return {"q": q.reshape(t, -1).to(dt), "k": kv.reshape(t, -1).to(dt), "v": vv.reshape(t, -1).to(dt)}


def _plain_attention(s):
    c = s["case"]
    hq, hk, d, page = c["hq"], c["hk"], c["d"], c["page"]
    lens, starts, n, nq = s["lens"].long(), s["starts"].long(), c["seqs"], s["max_q"]
    cnt = starts[1:] - starts[:-1]
    row = -(-s["max_len"] // page)
    groups = s["cache"][s["table"][:, :row].long()].transpose(1, 2).reshape(n, hk, -1, 16 * d + 128)
    kc, kp, vc, vp = _unpack_groups(groups, d)
    k, v = _values(kc, kp).reshape(n, hk, -1, d), _values(vc, vp).reshape(n, hk, -1, d)
    i = torch.arange(nq, device=DEV)
    at = (starts[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][at].float().view(n, nq, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d)
    score = (q @ k.transpose(-1, -2)).view(n, hq, nq, -1) * (1.0 / math.sqrt(d))
    pos = ((lens - cnt)[:, None] + i)[:, None, :, None]
    j = torch.arange(k.shape[2], device=DEV)
    see = (j <= pos) & (i < cnt[:, None])[:, None, :, None]
    if c["window"]:
        see = see & ((j > pos - c["window"]) | (j < c["sinks"]))
    score = score.masked_fill(~see, -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = (p.view(n, hk, -1, p.shape[-1]) @ v).view(n, hq, nq, d) / total.clamp_min(1e-30)
    lse = (top + torch.log(total))[..., 0]
    mine = i < cnt[:, None]
    return {"out": o.permute(0, 2, 1, 3)[mine].reshape(-1, hq * d).to(s["q"].dtype), "lse": lse.transpose(1, 2)[mine]}


def _plain_fp8(s):
    x, w, sw = s["x"].float(), s["w"], s["sw"]
    (m, k), n = x.shape, w.shape[0]
    kb = sw.shape[1]
    x = torch.cat([x, x.new_zeros(m, kb * 128 - k)], 1).view(m, kb, 128)
    sx = x.abs().amax(-1, keepdim=True) / 448.0
    xq = torch.where(sx > 0, x / sx, x).to(torch.float8_e4m3fn).float()
    xv = (xq * sx).view(m, -1)[:, :k]
    wv = w.float() * sw.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return (xv @ wv.t()).to(s["out"].dtype)


PLAIN = {"append": _plain_append, "attention": _plain_attention, "fp8": _plain_fp8}


# ------------------------------------------------------------------------------------ the library's calls


def _plan(s):
    """What a program keeps beside its buffers: descriptors and a workspace."""
    from paper_1911_08076_gb300 import ifq
    c = s["case"]
    types = {"f16": ifq.IFQ_F16, "bf16": ifq.IFQ_BF16, "f32": ifq.IFQ_F32}
    if c["do"] == "fp8":
        d = ifq.fp8_desc(c["m"], c["n"], c["k"], types[c["dtype"]], types[c["out"]])
        size = ifq.ifq_fp8_workspace_bytes(d)
    else:
        pool = ifq.kv4_cache(s["cache"].shape[0], c["page"], c["hk"], c["d"])
        if c["do"] == "append":
            rope = {"halves": ifq.IFQ_ROPE_HALVES, "pairs": ifq.IFQ_ROPE_PAIRS}[c["rope"]]
            wide = s["qkv"].shape[1]
            d = ifq.kv4_append_desc(pool, c["tokens"], c["hq"], types[c["dtype"]], rope, c["rot"], s["cos"].shape[0],
                                    q_stride=wide, k_stride=wide, v_stride=wide)
            return ifq, d, None, 0
        d = ifq.kv4_attention_desc(pool, c["seqs"], s["q"].shape[0], s["max_q"], s["table"].shape[1], c["hq"],
                                   types[c["dtype"]], 1.0 / math.sqrt(c["d"]), c["window"], c["sinks"],
                                   max_len=s["max_len"])
        size = ifq.ifq_kv4_attention_workspace_bytes(d)
    return ifq, d, torch.empty(max(size, 1), dtype=torch.uint8, device=DEV), size


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    ifq, d, ws, size = s["plan"]
    do = s["case"]["do"]
    if do == "append":
        ifq.ifq_kv4_append(d, s["q"], s["k"], s["v"], s["cos"], s["sin"], s["pos"], s["slots"], s["q_out"], s["cache"])
        ifq.ifq_kv4_read(d, s["cache"], s["slots"], s["k_out"], s["v_out"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if do == "attention":
        ifq.ifq_kv4_attention(d, s["q"], s["cache"], s["table"], s["lens"], s["starts"], s["out"], s["lse"], ws, size)
        return {"out": s["out"], "lse": s["lse"]}
    ifq.ifq_fp8_quantize(d, s["x"], s["xq"], s["sx"])
    ifq.ifq_fp8_matmul(d, s["xq"], s["sx"], s["w"], s["sw"], s["out"], ws, size)
    return s["out"]


def run(state):
    return _own(state) if own else PLAIN[state["case"]["do"]](state)


# ------------------------------------------------------------------------------------ work


def work(case):
    c = case
    if c["do"] == "append":
        t, size = c["tokens"], 2
        q, kv = t * c["hq"] * c["d"], t * c["hk"] * c["d"]
        held = t * c["hk"] * (c["d"] + 8)  # codes and parameters of both
        # rotated q; k and v in, the cache's bytes out; those in again, the values out; the tables' rows
        return {"bytes": 2 * q * size + 2 * kv * size + held + held + 2 * kv * size + t * (c["rot"] * 4 + 12 + 8),
                "flops": 3 * (q + kv) + 12 * kv}
    if c["do"] == "attention":
        n, mid = c["seqs"], (c["len_lo"] + c["len_hi"]) / 2
        nq = sum(c["nq"] - i * 5 % (c["nq"] // 2 + 1) for i in range(n)) / n
        span = min(mid, c["window"] + c["sinks"]) if c["window"] else mid - (nq - 1) / 2  # keys a query sees
        read = min(mid, c["window"] + c["sinks"] + nq) if c["window"] else mid           # keys a sequence reads
        rows = n * nq * c["hq"]
        return {"bytes": n * read * c["hk"] * (c["d"] + 8) + rows * (4 * c["d"] + 4) + 4 * n * read / c["page"],
                "flops": 4 * rows * span * c["d"]}
    m, n, k = c["m"], c["n"], c["k"]
    out = 4 if c["out"] == "f32" else 2
    return {"bytes": 2 * m * k + n * k + 4 * (-(-n // 128)) * (-(-k // 128)) + out * m * n, "flops": 2 * m * n * k}


# ------------------------------------------------------------------------------------ in 64 bits


def _exact_rows(x, cos, sin, c):
    """The rotation as a product with complex numbers."""
    rot = c["rot"]
    turn = torch.complex(cos, sin)[:, None]
    y = x.clone()
    if c["rope"] == "halves":
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_held(x):
    """The values that 4 bits leave of each row of x (float64)."""
    x = torch.clamp(x, -65504, 65504)
    lo, hi = torch.aminmax(x, dim=-1, keepdim=True)
    step, lo = ((hi - lo) / 15).half().double(), lo.half().double()
    return torch.where(step > 0, torch.clamp(torch.round((x - lo) / step), 0, 15), 0.0) * step + lo


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["do"] == "append":
        t, d, p = c["tokens"], c["d"], s["pos"].long()
        cos, sin = s["cos"].double()[p], s["sin"].double()[p]
        q = _exact_rows(s["q"].double().reshape(t, c["hq"], d), cos, sin, c)
        k = _exact_rows(s["k"].double().reshape(t, c["hk"], d), cos, sin, c)
        v = s["v"].double().reshape(t, c["hk"], d)
        return {"q": q.reshape(t, -1), "k": _exact_held(k).reshape(t, -1), "v": _exact_held(v).reshape(t, -1)}
    if c["do"] == "attention":
        hq, hk, d = c["hq"], c["hk"], c["d"]
        if 4.0 * c["seqs"] * c["nq"] * c["len_hi"] * hq * d > 4e12:
            return None
        starts, lens = s["starts"].tolist(), s["lens"].tolist()
        out = torch.zeros(starts[-1], hq, d, dtype=torch.float64, device=DEV)
        lse = torch.full((starts[-1], hq), -math.inf, dtype=torch.float64, device=DEV)
        for b, length in enumerate(lens):
            a, e = starts[b], starts[b + 1]
            if a == e or not length:
                continue
            ids = s["table"][b, :-(-length // c["page"])].long()
            pos = torch.arange(length - (e - a), length, device=DEV)[:, None]
            j = torch.arange(length, device=DEV)
            hide = j > pos
            if c["window"]:
                hide |= (j <= pos - c["window"]) & (j >= c["sinks"])
            for h in range(hk):
                kc, kp, vc, vp = (x.reshape(-1, x.shape[-1])[:length].double() for x in _unpack_groups(s["cache"][ids, h], d))
                k, v = kc * kp[:, :1] + kp[:, 1:], vc * vp[:, :1] + vp[:, 1:]
                for q0 in range(0, e - a, 256):
                    rows = slice(a + q0, min(a + q0 + 256, e))
                    q = s["q"][rows].double().view(-1, hq, d)[:, h * (hq // hk):(h + 1) * (hq // hk)]
                    x = torch.einsum("thd,jd->thj", q, k) / math.sqrt(d)
                    x.masked_fill_(hide[q0:q0 + 256, None], -math.inf)
                    l = torch.logsumexp(x, -1)
                    heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
                    lse[rows, heads] = l
                    out[rows, heads] = torch.einsum("thj,jd->thd", torch.exp(x - l[..., None]), v)
        return {"out": out.view(-1, hq * d), "lse": lse}
    x, sw = s["x"].double(), s["sw"].double()
    y = torch.zeros(c["m"], c["n"], dtype=torch.float64, device=DEV)
    for b in range(sw.shape[1]):
        cols = slice(128 * b, min(128 * b + 128, c["k"]))
        sx = (s["x"][:, cols].float().abs().amax(1, keepdim=True) / 448.0).double()
        xq = torch.where(sx > 0, x[:, cols] / sx, 0.0).float().to(torch.float8_e4m3fn).double()
        y += sx * (xq @ s["w"][:, cols].double().t()) * sw[:, b].repeat_interleave(128)[:c["n"]]
    return y
