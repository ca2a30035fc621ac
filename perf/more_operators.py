"""Performance cases of the operators around a quantised decoder's attention block.

Four groups, each reached through the binding's calls where `own` is true:

* matmul: a product with 4-bit weights (ifq_w4_matmul), with or without a residual added to it: from one token to a prompt;
* gated: both projections of a gated feed-forward block from 4-bit weights, the activation and the product (ifq_w4_gated);
* norm: a residual added and the root-mean-square norm of the sum (ifq_rms_norm);
* scores: log-probabilities of given tokens, the log-sum-exp, the entropy and the likeliest tokens of rows of logits
  (ifq_token_scores).

Where `own` is false run() computes the same in elementary torch operations in 32 bits.

The weights.  w[j][k] = code * scale + min rounded once to the weights' type, with codes of 4 bits and a scale and a minimum of
that type for each row and group of 32, 64 or 128 along k.  codes are uint8 [rows][k / 2], the even k in the low half of a
byte; scales and mins are [rows][ceil(k / group)].  The rows of a gated pair are the gate's, then the other's.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------ cases


def _matmul(name, m, n, k, group=128, dtype="bf16", out=None, residual=False):
    return {"name": name, "do": "matmul", "m": m, "n": n, "k": k, "group": group, "dtype": dtype, "out": out or dtype,
            "residual": residual}


def _gated(name, m, n, k, group=128, dtype="bf16", act="silu"):
    return {"name": name, "do": "gated", "m": m, "n": n, "k": k, "group": group, "dtype": dtype, "act": act}


def _norm(name, rows, dim, dtype="bf16", residual=True):
    return {"name": name, "do": "norm", "rows": rows, "dim": dim, "dtype": dtype, "residual": residual}


def _scores(name, rows, vocab, dtype="f32", top=0, scale=1.0):
    return {"name": name, "do": "scores", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "scale": scale}


def listed():
    return [
        # one token through an output projection, added to the residual: a latency-bound call
        _matmul("matmul_1x4096x4096", 1, 4096, 4096, residual=True),
        # the logits of a small batch: the largest weights of a model
        _matmul("matmul_8x131072x4096_head", 8, 131072, 4096, 64, out="f32"),
        # an odd batch of conversations, sizes that end inside tiles and a last group that is not full
        _matmul("matmul_41x6152x4112", 41, 6152, 4112, 32, "f16"),
        # a prompt through the second half of a feed-forward block
        _matmul("matmul_4096x4096x9216", 4096, 4096, 9216, residual=True),
        # one token through the first half of a feed-forward block
        _gated("gated_1x9216x4096", 1, 9216, 4096),
        # the tokens that a scheduler puts together in a step, odd sizes
        _gated("gated_333x5640x2064", 333, 5640, 2064, 64, "f16", "gelu_tanh"),
        # a prompt through it
        _gated("gated_2048x9216x4096", 2048, 9216, 4096),
        # one token between two blocks: a latency-bound call
        _norm("norm_1x4096", 1, 4096),
        # a prompt between two blocks
        _norm("norm_8191x4096", 8191, 4096),
        # one sampled token of one conversation
        _scores("scores_1x131072", 1, 131072, "f32", 20, 1.25),
        # a batch of conversations over an odd vocabulary
        _scores("scores_48x100003", 48, 100003, "bf16", 5),
        # a prompt's tokens scored, with a few alternatives each
        _scores("scores_2048x131072", 2048, 131072, "bf16", 8),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v if v <= 1024 else min(v | 1, hi)  # the large ones odd


def draw(rng):
    most = {"matmul": 6e9, "gated": 6e9, "norm": 2.6e8, "scores": 5e8}
    while True:
        do = rng.choice(["matmul", "matmul", "gated", "gated", "norm", "scores"])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        if do in ("matmul", "gated"):
            m, group = _log(rng, 1, 4096), rng.choice([32, 64, 128, 128])
            n = rng.choice([128 * 2 ** rng.randint(2, 6), _log(rng, 64, 16384)])
            k = rng.choice([128 * 2 ** rng.randint(2, 6), 8 * (2 * _log(rng, 8, 800) + 1)])
            if do == "matmul":
                c = _matmul("", m, n, k, group, dtype, rng.choice([dtype, dtype, "f32"]), rng.random() < 0.5)
            else:
                c = _gated("", m, n, k, group, dtype, rng.choice(["silu", "silu", "gelu", "gelu_tanh"]))
        elif do == "norm":
            c = _norm("", _log(rng, 1, 16384), 8 * _log(rng, 8, 2048), dtype, rng.random() < 0.7)
        else:
            c = _scores("", _log(rng, 1, 4096), _log(rng, 1000, 262144), rng.choice([dtype, "f32"]),
                        rng.choice([0, 1, 5, 20, 32]), rng.choice([1.0, 1.0, 0.7]))
        del c["name"]
        w = work(c)
        if max(w["bytes"], w["flops"] / 50) <= most[do]:
            return c


# ------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(191108 + seed)
    return g


def _quantised(g, rows, k, group, dtype):
    """Normal weights in 4 bits: codes, scales, mins."""
    groups = -(-k // group)
    codes = torch.empty(rows, k // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(rows, groups, dtype=dtype, device=DEV)
    mins = torch.empty_like(scales)
    step = max(1, (1 << 27) // (groups * group))
    for r in range(0, rows, step):
        w = torch.randn(min(step, rows - r), groups, group, generator=g, device=DEV) * 0.02
        lo = w.amin(-1)
        s, m = ((w.amax(-1) - lo) / 15.0).to(dtype), lo.to(dtype)
        c = torch.round((w - m.float()[..., None]) / s.float()[..., None]).clamp_(0.0, 15.0).to(torch.uint8).flatten(1)[:, :k]
        codes[r:r + step] = c[:, 0::2] | (c[:, 1::2] << 4)
        scales[r:r + step], mins[r:r + step] = s, m
    return codes, scales, mins


def _activations(g, m, k, dtype):
    x = torch.randn(m, k, generator=g, device=DEV)
    return (x * (1 + 8 * (torch.rand(k, generator=g, device=DEV) < 0.01))).to(dtype)  # a few loud channels


def _prepare_w4(c, g):
    m, n, k, dt = c["m"], c["n"], c["k"], TYPES[c["dtype"]]
    gated = c["do"] == "gated"
    s = {"x": _activations(g, m, k, dt)}
    s["codes"], s["scales"], s["mins"] = _quantised(g, 2 * n if gated else n, k, c["group"], dt)
    s["residual"] = (torch.randn(m, n, generator=g, device=DEV) * 2).to(TYPES[c["out"]]) if c.get("residual") else None
    s["out"] = torch.empty(m, n, dtype=dt if gated else TYPES[c["out"]], device=DEV)
    if own:
        from paper_1911_08076_gb300 import ifq
        code = {"f16": ifq.IFQ_F16, "bf16": ifq.IFQ_BF16, "f32": ifq.IFQ_F32}
        w = ifq.w4_weights(n, k, c["group"], code[c["dtype"]], gated)
        s["packed"] = torch.empty(ifq.ifq_w4_bytes(w), dtype=torch.uint8, device=DEV)
        ifq.ifq_w4_pack(w, s["codes"], s["scales"], s["mins"], s["packed"])
        act = {"silu": ifq.IFQ_ACT_SILU, "gelu": ifq.IFQ_ACT_GELU, "gelu_tanh": ifq.IFQ_ACT_GELU_TANH}
        s["desc"] = ifq.w4_desc(w, m, code[c["dtype"] if gated else c["out"]], act[c["act"]] if gated else 0)
    return s


def _prepare_norm(c, g):
    rows, dim, dt = c["rows"], c["dim"], TYPES[c["dtype"]]
    s = {"x": (torch.randn(rows, dim, generator=g, device=DEV) * 0.5).to(dt),
         "weight": (1 + 0.1 * torch.randn(dim, generator=g, device=DEV)).to(dt),
         "out": torch.empty(rows, dim, dtype=dt, device=DEV), "residual": None, "sum": None}
    if c["residual"]:  # the stream that the blocks add to: larger, with a few loud channels
        s["residual"], s["sum"] = _activations(g, rows, dim, dt), torch.empty(rows, dim, dtype=dt, device=DEV)
    if own:
        from paper_1911_08076_gb300 import ifq
        s["desc"] = ifq.norm_desc(rows, dim, ifq.IFQ_F16 if c["dtype"] == "f16" else ifq.IFQ_BF16, EPS)
    return s


def _prepare_scores(c, g):
    rows, vocab, top = c["rows"], c["vocab"], c["top"]
    logits = torch.empty(rows, vocab, dtype=TYPES[c["dtype"]], device=DEV)
    # a model's logits: a broad floor and a few tokens that stand out of it, more or less from row to row
    sharp = 1 + 3 * torch.rand(rows, 1, generator=g, device=DEV)
    step = max(1, (1 << 27) // vocab)
    for r in range(0, rows, step):
        z = torch.randn(min(step, rows - r), vocab, generator=g, device=DEV)
        logits[r:r + step] = z * sharp[r:r + step]
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    s = {"logits": logits, "tokens": tokens, "logprobs": torch.empty(rows, device=DEV),
         "lse": torch.empty(rows, device=DEV), "entropy": torch.empty(rows, device=DEV),
         "top_ids": torch.empty(rows, top, dtype=torch.int64, device=DEV), "top_logprobs": torch.empty(rows, top, device=DEV)}
    if own:
        from paper_1911_08076_gb300 import ifq
        code = {"f16": ifq.IFQ_F16, "bf16": ifq.IFQ_BF16, "f32": ifq.IFQ_F32}[c["dtype"]]
        s["desc"] = ifq.scores_desc(rows, vocab, code, top, c["scale"])
    return s


PREPARE = {"matmul": _prepare_w4, "gated": _prepare_w4, "norm": _prepare_norm, "scores": _prepare_scores}


def prepare(case, seed):
    s = PREPARE[case["do"]](case, _gen(seed))
    s["case"] = case
    if own:
        from paper_1911_08076_gb300 import ifq
        s["ifq"] = ifq
    return s


# ------------------------------------------------------------------------------------ the plain forms


def _weights(s, r0, r1):
    """Rows r0 to r1 of the weights as the values that they stand for, in float32."""
    c, k = s["case"], s["x"].shape[1]
    b = s["codes"][r0:r1]
    codes = torch.stack([b & 15, b >> 4], -1).view(len(b), k).float()
    at = torch.arange(k, device=DEV) // c["group"]
    w = codes * s["scales"][r0:r1].float()[:, at] + s["mins"][r0:r1].float()[:, at]
    return w.to(s["x"].dtype).float()


def _plain_matmul(s):
    y = s["x"].float() @ _weights(s, 0, len(s["codes"])).t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["out"].dtype)


def _plain_gated(s):
    c = s["case"]
    x, n = s["x"].float(), c["n"]
    a, b = x @ _weights(s, 0, n).t(), x @ _weights(s, n, 2 * n).t()
    if c["act"] == "silu":
        a = a / (1 + torch.exp(-a))
    elif c["act"] == "gelu":
        a = 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    else:
        a = a / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a)))
    return (a * b).to(s["out"].dtype)


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = (h + s["residual"].float()).to(s["x"].dtype).float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    out = {"out": y.to(s["x"].dtype)}
    if s["residual"] is not None:
        out["sum"] = h.to(s["x"].dtype)
    return out


def _plain_scores(s):
    c = s["case"]
    rows, vocab, top = c["rows"], c["vocab"], c["top"]
    parts = {k: [] for k in ("logprobs", "lse", "entropy", "top_ids", "top_logprobs")}
    step = max(1, (1 << 26) // vocab)
    for r in range(0, rows, step):
        raw = s["logits"][r:r + step]
        z = raw.float() * c["scale"]
        most = z.amax(-1, keepdim=True)
        d = z - most
        e = torch.exp(d)
        total = e.sum(-1, keepdim=True, dtype=torch.float64)
        lse = most + torch.log(total)
        parts["lse"].append(lse[:, 0].float())
        parts["entropy"].append((torch.log(total) - (e * d).sum(-1, keepdim=True, dtype=torch.float64) / total)[:, 0].float())
        parts["logprobs"].append((z.gather(1, s["tokens"][r:r + step, None]) - lse)[:, 0].float())
        if top:
            ids = torch.sort(raw, dim=-1, descending=True, stable=True)[1][:, :top]
            parts["top_ids"].append(ids)
            parts["top_logprobs"].append((z.gather(1, ids) - lse).float())
    return {k: torch.cat(v) for k, v in parts.items() if v}


PLAIN = {"matmul": _plain_matmul, "gated": _plain_gated, "norm": _plain_norm, "scores": _plain_scores}


# ------------------------------------------------------------------------------------ the calls


def _own_matmul(s):
    s["ifq"].ifq_w4_matmul(s["desc"], s["x"], s["packed"], s["out"], s["residual"])
    return s["out"]


def _own_gated(s):
    s["ifq"].ifq_w4_gated(s["desc"], s["x"], s["packed"], s["out"])
    return s["out"]


def _own_norm(s):
    s["ifq"].ifq_rms_norm(s["desc"], s["x"], s["residual"], s["weight"], s["sum"], s["out"])
    return {"out": s["out"], "sum": s["sum"]} if s["sum"] is not None else {"out": s["out"]}


def _own_scores(s):
    names = ("logprobs", "lse", "entropy", "top_ids", "top_logprobs") if s["case"]["top"] else ("logprobs", "lse", "entropy")
    s["ifq"].ifq_token_scores(s["desc"], s["logits"], s["tokens"], *[s[k] for k in names])
    return {k: s[k] for k in names}


OWN = {"matmul": _own_matmul, "gated": _own_gated, "norm": _own_norm, "scores": _own_scores}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["do"]](state)


# ------------------------------------------------------------------------------------ the least work


def work(case):
    c = case
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if c["do"] in ("matmul", "gated"):
        m, n, k = c["m"], c["n"], c["k"]
        rows = 2 * n if c["do"] == "gated" else n
        out = size[c.get("out", c["dtype"])]
        weights = rows * (k // 2 + 4 * -(-k // c["group"]))
        return {"bytes": weights + 2 * m * k + m * n * out * (2 if c.get("residual") else 1), "flops": 2 * m * rows * k}
    if c["do"] == "norm":
        rows, dim = c["rows"], c["dim"]
        return {"bytes": 2 * dim * (1 + rows * (4 if c["residual"] else 2)), "flops": (5 if c["residual"] else 4) * rows * dim}
    rows, vocab = c["rows"], c["vocab"]
    return {"bytes": rows * (vocab * size[c["dtype"]] + 8 + 12 + 12 * c["top"]), "flops": 6 * rows * vocab}


# ------------------------------------------------------------------------------------ in 64 bits


def _exact_products(c, s, first):
    """x times rows first to first + n of the weights, a group at a time: each group's products in float64."""
    m, n, k, size = c["m"], c["n"], c["k"], c["group"]
    y = torch.zeros(m, n, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // k)
    for r in range(0, n, step):
        rows = slice(first + r, first + min(r + step, n))
        count = rows.stop - rows.start
        w = torch.empty(count, k, dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = (s["codes"][rows] % 16).double(), (s["codes"][rows] // 16).double()
        for b in range(-(-k // size)):
            part = w[:, b * size:(b + 1) * size]
            part.mul_(s["scales"][rows, b:b + 1].double()).add_(s["mins"][rows, b:b + 1].double())
        w = w.to(s["x"].dtype).double()
        torch.mm(s["x"].double(), w.t(), out=y[:, r:r + count]) if n <= step else y[:, r:r + count].copy_(s["x"].double() @ w.t())
    return y


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["do"] == "matmul":
        y = _exact_products(c, s, 0)
        return y if s["residual"] is None else y + s["residual"].double()
    if c["do"] == "gated":
        a, b = _exact_products(c, s, 0), _exact_products(c, s, c["n"])
        if c["act"] == "silu":
            return a * torch.special.expit(a) * b
        if c["act"] == "gelu":
            return a * torch.special.ndtr(a) * b
        return 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))) * b
    if c["do"] == "norm":
        h = s["x"].double()
        out = {}
        if c["residual"]:
            out["sum"] = h + s["residual"].double()
            h = out["sum"].to(s["x"].dtype).double()   # what is normalised is the sum as it is kept
        out["out"] = h / torch.sqrt(h.square().sum(-1, keepdim=True) / c["dim"] + EPS) * s["weight"].double()
        return out
    out = {k: torch.empty(c["rows"], dtype=torch.float64, device=DEV) for k in ("logprobs", "lse", "entropy")}
    if c["top"]:
        out["top_ids"] = torch.empty(c["rows"], c["top"], dtype=torch.int64, device=DEV)
        out["top_logprobs"] = torch.empty(c["rows"], c["top"], dtype=torch.float64, device=DEV)
    step = max(1, (1 << 25) // c["vocab"])
    for r in range(0, c["rows"], step):
        z = s["logits"][r:r + step].double() * c["scale"]
        lp = torch.log_softmax(z, -1)
        at = slice(r, r + len(z))
        out["lse"][at] = torch.logsumexp(z, -1)
        out["entropy"][at] = -(lp.exp() * lp).sum(-1)
        out["logprobs"][at] = lp.gather(1, s["tokens"][at, None])[:, 0]
        if c["top"]:
            # the likeliest tokens one by one, the first of equals
            left = s["logits"][at].float()
            for i in range(c["top"]):
                best = (left == left.amax(-1, keepdim=True)).to(torch.uint8).argmax(-1, keepdim=True)
                out["top_ids"][at, i:i + 1], out["top_logprobs"][at, i:i + 1] = best, lp.gather(1, best)
                left.scatter_(1, best, -math.inf)
    return out
