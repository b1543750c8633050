"""Operators of the framework's narrow formats, each on its own: what they take, their plain forms, their definition.

  cache    rows of K and V quantised to 8 bits as they are written into a cache, and rows (or all of it) read back:
           Marche.scatter_kv_quantized + Marche.gather_kv_quantized
  attend   attention of active rows over a cache held in 8 bits, from a single token to every token:
           Marche.attention_quantized
  linear   projection of a few rows by a matrix held in 4 bits with scales per group: Marche.linear_quantized

A case's fields:

  kind      "cache", "attend" or "linear"        operand   type of the projections' operands and of attention's output
  batch, seq, heads, kv_heads, dim    samples, cached tokens per sample, query heads, cached heads, head_dim
  rows      cache: tokens written per sample; attend: query rows per sample; linear: rows
  read      cache: "rows" reads the written tokens back, "all" the whole cache
  fused     cache, attend: k, v and q are columns of one [rows][q | k | v] buffer, as the fused projection leaves them
  ragged    attend: a number of valid keys per sample, zero among them, instead of all of them
  out, in_, group, epilogue    linear: outputs, inputs, inputs per scale, MARCHE_EPI_* code
"""
from __future__ import annotations

import functools
import math

import torch

own = False

OPERAND = {"f16": torch.float16, "bf16": torch.bfloat16}
SCALE_PAD = 64          # rows of scales are padded to a multiple of this


def _cache(name, batch, seq, kv_heads, dim, rows, read, fused, operand="f16"):
    return dict(name=name, kind="cache", batch=batch, seq=seq, kv_heads=kv_heads, dim=dim, rows=rows, read=read, fused=fused,
                operand=operand)


def _attend(name, batch, seq, heads, kv_heads, dim, rows, ragged, fused, operand):
    return dict(name=name, kind="attend", batch=batch, seq=seq, heads=heads, kv_heads=kv_heads, dim=dim, rows=rows, ragged=ragged,
                fused=fused, operand=operand)


def _linear(name, rows, out, in_, group, epilogue, operand):
    return dict(name=name, kind="linear", rows=rows, out=out, in_=in_, group=group, epilogue=epilogue, operand=operand)


def listed():
    return [
        # one image with guidance late in a run: a handful of fresh rows, all latency
        _cache("cache_rows_one_image", 2, 320, 12, 64, 9, "rows", True),
        # 64 images with guidance, mid run, the widest heads of the configurations
        _cache("cache_rows_batch", 128, 320, 16, 80, 43, "rows", True),
        # the initial refresh of long sequences, and the cache read back whole
        _cache("cache_fill_long", 6, 8191, 16, 64, 8191, "all", False),
        # the smallest step of a run: one token and its guidance row
        _attend("attend_one_token", 2, 320, 12, 12, 64, 1, False, True, "f16"),
        # one image of 32 x 32 tokens with guidance
        _attend("attend_rows_one_image", 2, 1088, 16, 16, 64, 41, False, False, "f16"),
        # 64 images with guidance, mid run
        _attend("attend_rows_batch", 128, 320, 16, 16, 80, 43, False, True, "bf16"),
        # one token per sequence over long ragged caches, four query heads to a cached one
        _attend("attend_token_long", 4, 65521, 32, 8, 128, 1, True, False, "bf16"),
        # every token of 32 x 32 images: the initial refresh, and the baseline that recomputes everything
        _attend("attend_full", 32, 1088, 16, 16, 64, 1088, False, False, "f16"),
        # one image, the fused q, k, v projection
        _linear("linear_rows_one_image", 2, 2304, 768, 64, 0, "f16"),
        # the first MLP projection on the active rows of one image
        _linear("linear_mlp_rows", 18, 4096, 1024, 128, 2, "bf16"),
        # a single row, a matrix that fills the second-level cache
        _linear("linear_row_wide", 1, 16384, 8192, 64, 0, "bf16"),
        # 32 rows less one, the largest matrix
        _linear("linear_rows_wide", 31, 24576, 12288, 128, 1, "f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cache", "attend", "attend", "linear"])
    operand = rng.choice(["f16", "bf16"])
    if kind == "linear":
        while True:
            rows, out, in_ = _log(rng, 1, 32), 16 * _log(rng, 8, 1536), 64 * _log(rng, 2, 192)
            group = rng.choice([32, 64, 128])
            if in_ % group == 0:
                break
        c = _linear("", rows, out, in_, group, rng.choice([0, 1, 2]), operand)
    elif kind == "cache":
        dim, kv_heads, seq = rng.choice([64, 64, 80, 128]), rng.choice([2, 8, 12, 16]), _log(rng, 1, 8191)
        batch = _log(rng, 1, max(1, min(128, 6 * 8191 * 16 * 64 // (seq * kv_heads * dim))))
        rows = seq if rng.random() < 0.25 else _log(rng, 1, seq)
        c = _cache("", batch, seq, kv_heads, dim, rows, rng.choice(["rows", "all"]), rng.random() < 0.5, operand)
    else:
        dim, group = rng.choice([64, 64, 80, 128]), rng.choice([1, 1, 2, 4, 8])
        kv_heads, seq = rng.choice([2, 8, 12, 16]), _log(rng, 1, 65521)
        most = 4 * 65521 * 8 * 128                                        # cached values of K
        batch = _log(rng, 1, max(1, min(128, most // (seq * kv_heads * dim))))
        most = 32 * 16 * 1088 * 1088 * 64                                 # products of queries and keys
        rows = _log(rng, 1, max(1, min(seq, 1536, most // (batch * seq * kv_heads * group * dim))))
        c = _attend("", batch, seq, kv_heads * group, kv_heads, dim, rows, rng.random() < 0.4, rng.random() < 0.5, operand)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _channels(gen, n):
    """Channels of a trained projection differ in size."""
    return torch.exp(0.5 * _normal(gen, n))


def _quantise_rows(x):
    """[..., dim] bf16 -> codes int8, scales fp32 [...]: code = round(127 x / amax), scale = amax / 127, ties to even."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    codes = torch.where(amax > 0, torch.round(x * 127.0 / amax), torch.zeros_like(x))
    return codes.to(torch.int8), torch.div(amax, torch.full_like(amax, 127.0)).squeeze(-1)     # (a plain number's reciprocal would be multiplied by)


def _random_cache(gen, batch, seq, heads, dim):
    """codes int8 [2][batch][seq][heads * dim] and scales fp32 [2][batch][heads][seq, padded]."""
    codes = torch.empty(2, batch, seq, heads * dim, dtype=torch.int8, device="cuda")
    padded = -(-seq // SCALE_PAD) * SCALE_PAD
    scales = torch.full((2, batch, heads, padded), float("nan"), device="cuda")   # nothing is to read the padding
    for which in range(2):
        x = (_normal(gen, batch, seq, heads * dim) * _channels(gen, heads * dim)).to(torch.bfloat16)
        c, s = _quantise_rows(x.view(batch, seq, heads, dim))
        codes[which] = c.view(batch, seq, -1)
        scales[which, :, :, :seq] = s.transpose(1, 2)
    return codes, scales


def _quantise_matrix(w, group):
    """fp32 [out][in] -> codes int8 in -7 .. 7, scales bf16 [out][in / group]."""
    g = w.view(w.shape[0], -1, group)
    top = g.abs().amax(-1)
    scales = torch.div(top, torch.full_like(top, 7.0)).to(torch.bfloat16)
    s = scales.float().unsqueeze(-1)
    codes = torch.where(s > 0, torch.round(g / s).clamp(-7, 7), torch.zeros_like(g))
    return codes.to(torch.int8).view_as(w), scales


@functools.lru_cache(maxsize=None)
def _context(operand):
    """The context a program has; the operators take their sizes from their own arguments."""
    from paper_2506_12035_b200.binding import BLOCK_FIELDS, MATRIX_FIELDS, Marche, upload_weights
    blk = {n: torch.zeros(384 if "qkv" in n else 128, 128) if n in MATRIX_FIELDS else torch.zeros(384 if "qkv" in n else 128)
           for n in BLOCK_FIELDS}
    return Marche(L=1, E=0, D=128, H=2, F=128, S=64, B=1, dtype="bf16", weights=upload_weights([blk], "bf16", operand=operand))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if own:
        from paper_2506_12035_b200 import binding
        s["m"] = _context(case["operand"])
    if case["kind"] == "linear":
        M, N, K = case["rows"], case["out"], case["in_"]
        s["a"] = _normal(gen, M, K).to(OPERAND[case["operand"]])
        w = _normal(gen, N, K).mul_(K ** -0.5)
        s["bias"] = 0.1 * _normal(gen, N)
        s["codes"], s["scales"] = _quantise_matrix(w, case["group"])
        if case["epilogue"] == 1:
            s["residual"] = _normal(gen, M, N)
        if own:
            s["w"] = s["m"].quantize_weights(w, case["group"])
        return s
    B, S, Hkv, dh, n = case["batch"], case["seq"], case["kv_heads"], case["dim"], case["rows"]
    s["codes"], s["scales"] = _random_cache(gen, B, S, Hkv, dh)
    if own:
        s["cache"] = binding.QuantizedCache(s["codes"], s["scales"], Hkv)
    H, D = case.get("heads", Hkv), Hkv * dh
    qkv = torch.empty(B * n, H * dh + 2 * D if case["fused"] else max(H * dh, D), dtype=torch.bfloat16, device="cuda")
    if case["kind"] == "attend":
        qkv.copy_(_normal(gen, *qkv.shape))
        s["q"] = qkv[:, :H * dh]
        s["kv_len"] = None
        if case["ragged"]:
            lens = torch.randint(0, S + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            lens[0] = S
            if B > 2:
                lens[B // 2] = 0
            s["kv_len"] = lens
        if own:
            s["o"] = torch.empty(B * n, H * dh, dtype=OPERAND[case["operand"]], device="cuda")
        return s
    rows = (_normal(gen, 2, B * n, D) * _channels(gen, D)).to(torch.bfloat16)
    if case["fused"]:
        qkv.zero_()
        qkv[:, D:2 * D], qkv[:, 2 * D:] = rows[0], rows[1]
        s["k"], s["v"] = qkv[:, D:2 * D], qkv[:, 2 * D:]
    else:
        s["k"], s["v"] = rows[0], rows[1]
    s["idx"] = None
    if n < S:                                    # distinct tokens in random order; every token: in their own order
        s["idx"] = torch.rand(B, S, generator=gen, device="cuda").argsort(1)[:, :n].to(torch.int32).contiguous()
    n_read = S if case["read"] == "all" else n
    if own:
        s["back"] = torch.empty(2, B * n_read, D, dtype=torch.bfloat16, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _run_own(s)
    return {"cache": _plain_cache, "attend": _plain_attend, "linear": _plain_linear}[s["kind"]](s)


def _run_own(s):
    m = s["m"]
    if s["kind"] == "linear":
        if s["epilogue"] == 1:
            out = s["residual"].clone()
        else:
            out = torch.empty(s["rows"], s["out"], dtype=torch.bfloat16 if s["epilogue"] == 0 else OPERAND[s["operand"]], device="cuda")
        m.linear_quantized(s["a"], s["w"], s["bias"], s["epilogue"], out)
        return out
    if s["kind"] == "attend":
        m.attention_quantized(s["q"], s["q"].stride(0), s["rows"], s["heads"], s["cache"], s["kv_len"], s["o"])
        return s["o"]
    m.scatter_kv_quantized(s["k"], s["v"], s["k"].stride(0), s["idx"], s["rows"], s["cache"])
    whole = s["read"] == "all"
    m.gather_kv_quantized(s["cache"], None if whole else s["idx"], s["seq"] if whole else s["rows"], s["back"][0], s["back"][1],
                          s["back"].stride(1))
    return s["back"]


def _plain_cache(s):
    B, S, H, dh, n = s["batch"], s["seq"], s["kv_heads"], s["dim"], s["rows"]
    codes, scales = s["codes"].view(2, B, S, H, dh), s["scales"]
    at = torch.arange(S, device="cuda").expand(B, S) if s["idx"] is None else s["idx"].long()
    b = torch.arange(B, device="cuda").unsqueeze(1)
    c, t = _quantise_rows(torch.stack([s["k"], s["v"]]).view(2, B, n, H, dh))
    codes[:, b, at] = c
    scales.transpose(2, 3)[:, b, at] = t
    if s["read"] == "all":
        back = codes.float() * scales[..., :S].transpose(2, 3).unsqueeze(-1)
    else:
        back = codes[:, b, at].float() * scales.transpose(2, 3)[:, b, at].unsqueeze(-1)
    return back.to(torch.bfloat16).view(2, -1, H * dh)


def _plain_attend(s):
    B, S, H, Hkv, dh, n = s["batch"], s["seq"], s["heads"], s["kv_heads"], s["dim"], s["rows"]
    G = H // Hkv
    kv = s["codes"].view(2, B, S, Hkv, dh).permute(0, 1, 3, 2, 4).float() * s["scales"][..., :S].unsqueeze(-1)   # [2][B][Hkv][S][dh]
    q = s["q"].float().view(B, n, Hkv, G, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, dh)
    logits = q @ kv[0].transpose(-1, -2) * dh ** -0.5
    if s["kv_len"] is not None:
        there = torch.arange(S, device="cuda") < s["kv_len"].view(B, 1, 1, 1)
        logits = logits.masked_fill(~there, float("-inf"))
    top = logits.amax(-1, keepdim=True).clamp_min(-3e38)          # a sample without keys has none
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    o = p @ kv[1] / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(B, Hkv, G, n, dh).permute(0, 3, 1, 2, 4).reshape(B * n, H * dh).to(OPERAND[s["operand"]])


def _plain_linear(s):
    w = (s["codes"].view(s["out"], -1, s["group"]).float() * s["scales"].float().unsqueeze(-1)).view(s["out"], -1)
    y = s["a"].float() @ w.t() + s["bias"]
    if s["epilogue"] == 1:
        return s["residual"] + y
    if s["epilogue"] == 2:
        return (0.5 * y * (1.0 + torch.erf(y * 0.5 ** 0.5))).to(OPERAND[s["operand"]])
    return y.to(torch.bfloat16)


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        y = s["bias"].double().expand(s["rows"], -1).clone()
        for g in range(s["in_"] // s["group"]):
            cols = slice(g * s["group"], (g + 1) * s["group"])
            y += (s["a"][:, cols].double() @ s["codes"][:, cols].double().t()) * s["scales"][:, g].double()
        return s["residual"].double() + y if s["epilogue"] == 1 else 0.5 * y * torch.erfc(-y / math.sqrt(2.0)) if s["epilogue"] == 2 else y
    B, S, Hkv, dh, n = s["batch"], s["seq"], s["kv_heads"], s["dim"], s["rows"]
    if case["kind"] == "cache":
        fresh = []
        for x in (s["k"], s["v"]):
            x = x.double().reshape(B, n, Hkv, dh)
            top = x.abs().max(-1, keepdim=True).values
            step = (top / 127).float().double()                   # the scale is kept in 32 bits
            fresh.append((torch.round(x * 127 / top.clamp_min(1e-300)) * step).view(B, n, -1))
        if case["read"] == "rows":
            return torch.stack([x.view(B * n, -1) for x in fresh])
        whole = []
        for which in range(2):
            y = s["codes"][which].double().view(B, S, Hkv, dh) * s["scales"][which, :, :, :S].double().transpose(1, 2).unsqueeze(-1)
            y = y.view(B, S, -1)
            at = torch.arange(S, device="cuda").repeat(B, 1) if s["idx"] is None else s["idx"].long()
            y.scatter_(1, at.unsqueeze(-1).expand(-1, -1, Hkv * dh), fresh[which])
            whole.append(y.view(B * S, -1))
        return torch.stack(whole)
    H = s["heads"]
    out = torch.zeros(B, n, H, dh, dtype=torch.float64, device="cuda")
    q = s["q"].double().reshape(B, n, H, dh)
    for b in range(B):
        length = S if s["kv_len"] is None else int(s["kv_len"][b])
        if length == 0:
            continue
        k, v = ((s["codes"][w, b, :length].view(length, Hkv, dh).double() * s["scales"][w, b, :, :length].t().double().unsqueeze(-1))
                .transpose(0, 1).repeat_interleave(H // Hkv, 0) for w in range(2))        # [H][length][dh]
        p = torch.softmax(torch.matmul(q[b].transpose(0, 1), k.transpose(1, 2)) / math.sqrt(dh), -1)
        out[b] = torch.matmul(p, v).transpose(0, 1)
    return out.view(B * n, H * dh)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "linear":
        M, N, K = c["rows"], c["out"], c["in_"]
        rows_out = M * N * (8 if c["epilogue"] == 1 else 2)
        return {"bytes": N * K // 2 + N * K // c["group"] * 2 + M * K * 2 + N * 4 + rows_out, "flops": 2 * M * N * K}
    B, S, Hkv, dh, n = c["batch"], c["seq"], c["kv_heads"], c["dim"], c["rows"]
    token = Hkv * (dh + 4)                                        # one token of K or of V in the cache
    if c["kind"] == "cache":
        n_read = S if c["read"] == "all" else n
        left = n_read - n                                         # read, and not just written
        return {"bytes": 2 * B * (n * Hkv * dh * 2 + n * token + left * token + n_read * Hkv * dh * 2) + (4 * B * n if n < S else 0),
                "flops": 2 * B * Hkv * dh * (3 * n + n_read)}
    # ragged: lengths are uniform in 0 .. S, but for one full and one empty sample
    keys = B * S if not c["ragged"] else S + (B - 1 - (B > 2)) * S // 2
    return {"bytes": 2 * keys * token + 2 * 2 * B * n * c["heads"] * dh, "flops": 4 * n * c["heads"] * dh * keys}
