"""The 8-bit cache (write, read back, attention) and projections by 4-bit weights against plain computations in 64 bits.

Tolerances are bounds, from the roundings that the kernels make:
  codes, scales, values read back   none: equal bit by bit to the definition
  attention   o is a mean of values v with weights p; what is rounded is p vs (fp16: half a step is 2^-11 of it) and the result
              (half a step of its type), so |err| <= 2^-11 A + half |o| with A = sum p |v| / sum p; logits, exponentials and sums in fp32
              add less than 2^-13 A at these sizes (logits of |x| < 2^5: 2^-18 of p at most by x's own rounding and the products' sums).
              fp16 ends: a weight far below the largest is a subnormal, off by up to 2^-25 of its unit, which is 2^-7 of a power of two
              2^e that is at most twice the largest value scale, vmax / 127, of the (sample, head).  A key's term p v is then off by
              2^-25 2^-7 (2 vmax / 127) 127 = 2^-31 vmax, S keys' by S 2^-31 vmax, and the sum of weights that all is divided by is
              at least 1, the weight of the key that the reference is.  (It shows where A is nothing beside vmax: a column in which
              the one key that counts holds a zero.)
  linear      products are exact; sums of a group (8 steps of the tensor core, 2^-23 each, which may truncate) and of groups and
              warps (2^-24 each) are relative to sum |a w|; then half a step of the output's type; GELU's slope is below 1.13
"""
import numpy as np
import pytest
import torch

import synth
from helpers import make_model
from paper_2506_12035_b200 import binding
from paper_2506_12035_b200.binding import MarcheError, QuantizedCache

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def models():
    cfg = synth.CONFIGS["tiny"].replace(L=1, E=0, D=128, H=2, F=128, S=64, B=1, dtype="bf16", n_buffer=0)
    blocks = synth.make_weights(cfg)
    return {o: make_model(cfg, blocks, operand=o) for o in TYPES}


@pytest.fixture(autouse=True)
def no_wait_gave_up(models):
    yield
    for m in models.values():
        m.check_status()


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def definition(x):
    """[..., dh] bf16 -> codes (float64 whole numbers), scales fp32, as the header defines them."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    codes = torch.where(bad | (amax == 0), torch.zeros_like(x), torch.round(x * 127 / torch.where(amax > 0, amax, torch.ones_like(amax))))
    scales = (amax / 127).float()                                     # (no rounding of 53 bits comes near a tie of 24: amax has 8)
    return codes, torch.where(bad, torch.full_like(scales, float("nan")), scales).squeeze(-1)


def filled_cache(m, gen, B, S, H, dh, spread=True):
    """A cache with every row written by the definition; the padding of the scales is NaN."""
    cache = m.alloc_quantized_cache(B, S, H, dh)
    cache.scales.fill_(float("nan"))
    for which in range(2):
        x = randn(gen, B, S, H, dh)
        if spread:
            x = x * torch.exp(0.7 * randn(gen, B, S, H, 1))
        c, s = definition(x.to(torch.bfloat16))
        cache.codes[which] = c.to(torch.int8).view(B, S, -1)
        cache.scales[which, :, :, :S] = s.transpose(1, 2)
    return cache


def values(cache):
    """float64 [2][B][S][H][dh]"""
    c = cache.codes.double().view(2, cache.B, cache.S, cache.n_kv_heads, cache.head_dim)
    return c * cache.scales[..., :cache.S].double().transpose(2, 3).unsqueeze(-1)


# ------------------------------------------------------------------ write and read back
def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0)) and torch.equal(a.isnan(), b.isnan())


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("B,S,H,n", [(1, 1, 1, 1), (2, 320, 12, 9), (3, 65, 3, 64), (2, 67, 5, 67), (5, 33, 16, 1), (1, 4099, 2, 1500)])
def test_rows_written_and_read_back(models, dh, B, S, H, n):
    m, gen, D = models["f16"], gen_of(dh + S), H * dh
    cache = filled_cache(m, gen, B, S, H, dh)
    before_c, before_s = cache.codes.clone(), cache.scales.clone()
    ld = 3 * D + 8                                                   # columns of wider rows
    rows = (randn(gen, B * n, ld) * torch.exp(2 * randn(gen, B * n, 1))).to(torch.bfloat16)
    rows[0] = 0                                                      # a head of zeros
    rows[-1, D:] = torch.tensor([1.0, -0.5, 0.5, 254.0, 127.0, -127.0, 1.5, -1.0], device="cuda").repeat(ld)[:ld - D]   # ties: 63.5, 0.5
    k, v = rows[:, D:2 * D], rows[:, 2 * D:3 * D]
    idx = torch.rand(B, S, generator=gen, device="cuda").argsort(1)[:, :n].to(torch.int32).contiguous()
    idx[B - 1, n // 2] = -1                                          # left out
    idx[0, n - 1] = S                                                # out of range: left out
    m.scatter_kv_quantized(k, v, ld, idx, n, cache)
    want_c, want_s = before_c.view(2, B, S, H, dh).clone(), before_s.clone()
    for which, x in enumerate((k, v)):
        c, s = definition(x.reshape(B, n, H, dh))
        for b in range(B):
            there = (idx[b] >= 0) & (idx[b] < S)
            at = idx[b][there].long()
            want_c[which, b, at] = c[b][there].to(torch.int8)
            want_s[which, b][:, at] = s[b][there].t()
    assert torch.equal(cache.codes.view_as(want_c), want_c)
    assert same(cache.scales, want_s)
    # the same rows, and the whole of it, back
    ld_out = D + 16
    back = torch.full((2, B * n, ld_out), 7.0, dtype=torch.bfloat16, device="cuda")
    m.gather_kv_quantized(cache, idx, n, back[0], back[1], ld_out)
    val = values(cache).float().to(torch.bfloat16).view(2, B, S, D)  # (code * scale is exact in 64 bits; once to fp32, as the kernel does)
    for which in range(2):
        for b in range(B):
            for j in ([0, n // 2, n - 1] if n > 40 else range(n)):
                row, t = back[which, b * n + j], int(idx[b, j])
                want = val[which, b, t] if 0 <= t < S else torch.full((D,), 7.0, dtype=torch.bfloat16, device="cuda")
                assert torch.equal(row[:D], want) and bool((row[D:] == 7).all())
    whole = torch.full((2, B * S, D), 7.0, dtype=torch.bfloat16, device="cuda")
    m.gather_kv_quantized(cache, None, S, whole[0], whole[1], D)
    assert torch.equal(whole.view(2, B, S, D), val)


def test_values_at_the_ends_of_the_range(models):
    """The largest and smallest bf16 numbers, zeros of both signs, infinities and NaN: by the definition, head by head."""
    m, B, S, H, dh = models["bf16"], 1, 8, 2, 64
    cache = m.alloc_quantized_cache(B, S, H, dh)
    x = torch.ones(S, H, dh, device="cuda")
    x[0, 0] *= 3.38e38
    x[0, 0, 1], x[0, 0, 2] = -1.69e38, 1e36
    x[1, 0] *= 1e-40                                                  # subnormal
    x[2, 0] = -0.0
    x[3, 0, 5] = float("inf")
    x[4, 0, 6] = float("nan")
    x[5, 0, 7] = float("-inf")
    x[6, 0] *= 2.0 ** 119
    x = x.to(torch.bfloat16)
    rows = x.view(S, -1).contiguous()
    m.scatter_kv_quantized(rows, rows, H * dh, None, S, cache)
    c, s = definition(x)
    assert torch.equal(cache.codes[0, 0].view(S, H, dh), c.to(torch.int8))
    assert same(cache.scales[0, 0, :, :S], s.t().contiguous())
    out = torch.empty(2, S, H * dh, dtype=torch.bfloat16, device="cuda")
    m.gather_kv_quantized(cache, None, S, out[0], out[1], H * dh)
    bad = out[1].view(S, H, dh).isnan()
    assert bool(bad[3:6, 0].all()) and int(bad.sum()) == 3 * dh


def test_prefix_written_without_index(models):
    m, gen, B, S, H, dh, n = models["f16"], gen_of(1), 3, 50, 2, 64, 20
    cache = m.alloc_quantized_cache(B, S, H, dh)
    rows = randn(gen, 2, B * n, H * dh).to(torch.bfloat16)
    m.scatter_kv_quantized(rows[0], rows[1], H * dh, None, n, cache)
    c, _ = definition(rows.view(2, B, n, H, dh))
    assert torch.equal(cache.codes[:, :, :n].reshape(c.shape), c.to(torch.int8)) and not cache.codes[:, :, n:].any()


# ------------------------------------------------------------------ attention
def reference(cache, q, n, heads, kv_len):
    """o, the mean magnitude A and S 2^-31 vmax, float64 [B*n][heads][dh]."""
    B, S, Hkv, dh = cache.B, cache.S, cache.n_kv_heads, cache.head_dim
    kv = values(cache)
    q = q.double().reshape(B, n, heads, dh)
    o, A, low = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    for b in range(B):
        length = S if kv_len is None else min(max(int(kv_len[b]), 0), S)
        if length == 0:
            continue
        for h in range(heads):
            k, v = kv[0, b, :length, h * Hkv // heads], kv[1, b, :length, h * Hkv // heads]
            p = torch.softmax(q[b, :, h] @ k.t() / dh ** 0.5, -1)
            o[b, :, h], A[b, :, h], low[b, :, h] = p @ v, p @ v.abs(), length * 2.0 ** -31 * v.abs().max()
    return o.view(B * n, heads, dh), A.view(B * n, heads, dh), low.view(B * n, heads, dh)


KERNELS = {"auto": binding.ATTENTION_AUTO, "mma": binding.ATTENTION_MMA, "tcgen05": binding.ATTENTION_TCGEN05}


@pytest.fixture(params=["mma", "tcgen05"])
def both_kernels(request, models):
    """Each attention kernel asked for by name."""
    for m in models.values():
        m.set_tuning(attention_kernel=KERNELS[request.param])
    yield request.param
    for m in models.values():
        m.set_tuning(attention_kernel=binding.ATTENTION_AUTO)


def attend(m, cache, q, ld, n, heads, kv_len, o=None):
    o = torch.full((cache.B * n, heads * cache.head_dim), 7.0, dtype=m.operand_dtype, device="cuda") if o is None else o
    m.attention_quantized(q, ld, n, heads, cache, kv_len, o)
    return o


def assert_attention(o, cache, q, n, heads, kv_len):
    want, A, low = reference(cache, q, n, heads, kv_len)
    err = (o.double().view_as(want) - want).abs()
    limit = (2.0 ** -11 + 2.0 ** -13) * A + low + HALF[o.dtype] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -24   # (fp16's smallest steps)
    worst = (err / limit.clamp_min(1e-30)).max()
    assert bool((err <= limit).all()), "error %.3g of the bound" % float(worst)


SHAPES = [  # B, S, heads, cached heads, rows
    (2, 1, 4, 4, 1), (2, 2, 4, 4, 3), (1, 63, 3, 3, 5), (2, 64, 2, 2, 16), (3, 65, 2, 2, 17), (2, 320, 12, 12, 1), (2, 333, 12, 12, 41),
    (1, 257, 2, 2, 257), (20, 320, 16, 16, 43), (40, 129, 8, 8, 33), (1, 1088, 4, 4, 150), (2, 700, 16, 4, 1), (2, 700, 8, 1, 7),
    (1, 5003, 2, 2, 1), (1, 4999, 4, 2, 30), (3, 2500, 6, 6, 65), (33, 200, 16, 16, 129)]


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("B,S,heads,kv_heads,n", SHAPES)
def test_attention(models, both_kernels, dh, operand, B, S, heads, kv_heads, n):
    m, gen = models[operand], gen_of(S + n + dh)
    cache = filled_cache(m, gen, B, S, kv_heads, dh)
    ld = heads * dh + 24
    rows = randn(gen, B * n, ld).to(torch.bfloat16)
    q = rows[:, 8:8 + heads * dh]
    o = attend(m, cache, q, ld, n, heads, None)
    assert_attention(o, cache, q, n, heads, None)
    assert torch.equal(o, attend(m, cache, q, ld, n, heads, None))    # bit-reproducible


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("B,S,heads,kv_heads,n", [(150, 70, 2, 2, 50), (1, 130, 300, 150, 70), (7, 200, 16, 16, 300), (300, 320, 2, 2, 20)])
def test_attention_of_many_items(models, both_kernels, dh, B, S, heads, kv_heads, n):
    """More units than SMs and streams: several turns, full and short last tiles, samples of all lengths among them."""
    m, gen = models["f16"], gen_of(B + S + dh)
    cache = filled_cache(m, gen, B, S, kv_heads, dh)
    kv_len = torch.randint(-1, S + 2, (B,), generator=gen, device="cuda", dtype=torch.int32)
    q = randn(gen, B * n, heads * dh).to(torch.bfloat16)
    for lens in (None, kv_len):
        o = attend(m, cache, q, heads * dh, n, heads, lens)
        some = torch.randperm(B, generator=gen, device="cuda")[:4].tolist()
        for b in some:
            part = QuantizedCache(cache.codes[:, b:b + 1].contiguous(), cache.scales[:, b:b + 1].contiguous(), kv_heads)
            rows = slice(b * n, (b + 1) * n)
            assert_attention(o[rows], part, q[rows], n, heads, None if lens is None else lens[b:b + 1])
        assert torch.equal(o, attend(m, cache, q, heads * dh, n, heads, lens))


@pytest.mark.parametrize("dh,n,heads", [(64, 1, 4), (80, 40, 4), (128, 3, 8), (64, 150, 4)])
@pytest.mark.parametrize("lens", [[0, 1, 63, 64, 65, 700], [700, -5, 9999, 2, 0, 640], [0, 0, 0, 0, 0, 0]])
def test_samples_of_different_lengths(models, both_kernels, dh, n, heads, lens):
    """Keys behind a sample's length are not looked at (their scales are NaN here); none at all: zeros."""
    m, gen, B, S, kv = models["bf16"], gen_of(n), 6, 700, 4
    cache = filled_cache(m, gen, B, S, kv, dh)
    for b, length in enumerate(lens):
        cache.scales[:, b, :, max(min(length, S), 0):] = float("nan")
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = randn(gen, B * n, heads * dh).to(torch.bfloat16)
    o = attend(m, cache, q, heads * dh, n, heads, kv_len)
    cache.scales.nan_to_num_(nan=0.0)
    assert_attention(o, cache, q, n, heads, kv_len)
    for b, length in enumerate(lens):
        if length <= 0:
            assert not o.view(B, -1)[b].any()


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("n", [1, 20, 140])
def test_peaked_rows_and_scales_far_apart(models, both_kernels, dh, n):
    """Logits of tens, and keys whose value scales lie up to 2^40 apart, in both orders: the weight that counts keeps its bits."""
    m, gen, B, S, H = models["f16"], gen_of(n + dh), 2, 400, 2
    cache = filled_cache(m, gen, B, S, H, dh, spread=False)
    cache.scales[0, :, :, :S] *= 3.0
    cache.scales[1, 0, :, :S] *= torch.exp2(torch.linspace(-30, 10, S, device="cuda"))
    cache.scales[1, 1, :, :S] *= torch.exp2(torch.linspace(10, -30, S, device="cuda"))
    q = (2.0 * randn(gen, B * n, H * dh)).to(torch.bfloat16)
    o = attend(m, cache, q, H * dh, n, H, None)
    want, A, low = reference(cache, q, n, H, None)
    # sums of |q k| reach 2^9 here: the fp32 logits are off by up to 2^9 2^-20, and every weight by twice that share
    limit = (2.0 ** -11 + 2.0 ** -9.5) * A + low + HALF[o.dtype] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -24
    assert bool(((o.double().view_as(want) - want).abs() <= limit).all())


def test_query_rows_of_any_size(models, both_kernels):
    """A row of zeros weighs all keys alike; rows near the ends of bf16's range stay finite where the result is."""
    m, gen, B, S, H, dh, n = models["bf16"], gen_of(3), 1, 100, 1, 64, 20
    cache = filled_cache(m, gen, B, S, H, dh)
    q = randn(gen, n, dh)
    q[0] = 0
    q[1] *= 1e-39
    q[2] *= 1e-30
    q = q.to(torch.bfloat16)
    o = attend(m, cache, q, dh, n, H, None)
    assert_attention(o, cache, q, n, H, None)
    cache.scales[0] *= 1e-37
    q[3:] = (q[3:].float() * 1e37).to(torch.bfloat16)
    o = attend(m, cache, q, dh, n, H, None)
    assert_attention(o[3:], cache, q[3:], n - 3, H, None)


def test_a_key_that_is_not_a_number_reaches_its_sample_and_head_only(models, both_kernels):
    m, gen, B, S, H, dh, n = models["f16"], gen_of(4), 2, 130, 2, 64, 5
    cache = filled_cache(m, gen, B, S, H, dh)
    cache.scales[0, 1, 0, 129] = float("nan")
    q = randn(gen, B * n, H * dh).to(torch.bfloat16)
    bad = attend(m, cache, q, H * dh, n, H, None).view(B, n, H, dh).isnan()
    assert bool(bad[1, :, 0].all()) and int(bad.sum()) == n * dh


def test_a_cache_beyond_32_bit_offsets(models, both_kernels):
    """2^31 codes lie in front of V's last rows: written, read back and attended there."""
    m, gen, B, S, H, dh, n = models["bf16"], gen_of(5), 1, (1 << 20) + 77, 16, 80, 4
    cache = m.alloc_quantized_cache(B, S, H, dh)
    assert cache.codes.numel() > 1 << 31
    idx = torch.tensor([[0, 5, S - 2, S - 1]], dtype=torch.int32, device="cuda")
    rows = randn(gen, 2, n, H * dh).to(torch.bfloat16)
    m.scatter_kv_quantized(rows[0], rows[1], H * dh, idx, n, cache)
    back = torch.empty_like(rows)
    m.gather_kv_quantized(cache, idx, n, back[0], back[1], H * dh)
    c, s = definition(rows.view(2, n, H, dh))
    assert torch.equal(back.view(2, n, H, dh), (c * s.double().unsqueeze(-1)).float().to(torch.bfloat16))
    # all but these rows have logit 0 and value 0
    q = (8 * rows[0]).contiguous()
    o = attend(m, cache, q, H * dh, n, H, None).double().view(n, H, dh)
    k, v = (c * s.double().unsqueeze(-1))
    x = torch.einsum("nhd,khd->nhk", q.double().view(n, H, dh), k) / dh ** 0.5
    top = x.amax(-1, keepdim=True).clamp_min(0)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True) + (S - n) * torch.exp(-top)
    want, A = torch.einsum("nhk,khd->nhd", p, v) / total, torch.einsum("nhk,khd->nhd", p, v.abs()) / total
    # sums of |q k| reach 2^10: logits off by up to 2^10 2^-20; a million exponentials of the others add up in fp32, S / 64 in turn at most
    limit = (2.0 ** -11 + 2.0 ** -8) * A + HALF[torch.bfloat16] * want.abs() + 2.0 ** -40
    assert bool(((o - want).abs() <= limit).all())


def test_attention_on_a_stream_and_in_a_graph(models, both_kernels):
    """Two captured calls that share nothing but the context, replayed with new inputs in the same buffers."""
    m, gen, B, S, H, dh = models["f16"], gen_of(6), 2, 1500, 4, 64
    cache = filled_cache(m, gen, B, S, H, dh)
    q1, q2 = (randn(gen, B * n, H * dh).to(torch.bfloat16) for n in (1, 50))
    rows, idx = randn(gen, 2, B, H * dh).to(torch.bfloat16), torch.full((B, 1), 3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, b = attend(m, cache, q1, H * dh, 1, H, None), attend(m, cache, q2, H * dh, 50, H, None)
    side.synchronize()
    assert_attention(a, cache, q1, 1, H, None)
    assert_attention(b, cache, q2, 50, H, None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.scatter_kv_quantized(rows[0], rows[1], H * dh, idx, 1, cache)
        attend(m, cache, q1, H * dh, 1, H, None, a)
        attend(m, cache, q2, H * dh, 50, H, None, b)
    for token in (0, 700, 1499):
        rows.copy_(randn(gen, 2, B, H * dh))
        idx.fill_(token)
        q1.copy_(randn(gen, *q1.shape))
        graph.replay()
        torch.cuda.synchronize()
        c, _ = definition(rows.view(2, B, H, dh))
        assert torch.equal(cache.codes[:, :, token].view(2, B, H, dh), c.to(torch.int8))
        assert_attention(a, cache, q1, 1, H, None)
        assert_attention(b, cache, q2, 50, H, None)


# ------------------------------------------------------------------ weights of 4 bits
def unpack(w):
    """codes [N][K] and scales [N][K / group] of a QuantizedWeights, from the header's words."""
    N, K = w.N, w.K
    words = w.codes.cpu().numpy().view(np.uint32).reshape(N // 16, K // 64, 32, 4).astype(np.int64)
    codes = np.zeros((N, K), np.int64)
    tile, chunk, lane, s = np.indices(words.shape)
    g, t = lane // 4, lane % 4
    for r in range(4):
        for e in range(2):
            codes[16 * tile + g + 8 * (r % 2), 64 * chunk + 32 * (s // 2) + 8 * t + 4 * (s % 2) + 2 * (r // 2) + e] = (words >> (4 * r + 16 * e) & 15) - 8
    scales = w.scales.float().cpu().view(N // 16, K // w.group, 8, 2).permute(0, 3, 2, 1).reshape(N, -1)
    return torch.from_numpy(codes).cuda(), scales.cuda()


def matrix(gen, N, K):
    w = randn(gen, N, K) * torch.exp(randn(gen, N, 1)) * K ** -0.5
    w[0] = 0
    return w


@pytest.mark.parametrize("N,K,group", [(16, 64, 32), (16, 64, 64), (48, 192, 64), (32, 256, 128), (768, 768, 32), (2304, 768, 128)])
def test_weights_are_quantised_by_their_definition(models, N, K, group):
    m, gen = models["f16"], gen_of(N + K)
    w = matrix(gen, N, K)
    w[1, :group] = 3.5 * torch.arange(group, device="cuda") % 7       # ties
    codes, scales = unpack(m.quantize_weights(w, group))
    grouped = w.view(N, -1, group)
    top = grouped.abs().amax(-1)
    want_s = torch.div(top, torch.full_like(top, 7.0)).to(torch.bfloat16).float()     # (torch multiplies by a plain number's reciprocal)
    s = want_s.unsqueeze(-1)
    want = torch.where(s > 0, torch.round(grouped / torch.where(s > 0, s, torch.ones_like(s))).clamp(-7, 7), torch.zeros_like(grouped))
    assert torch.equal(scales, want_s) and torch.equal(codes, want.long().view(N, K))


def assert_linear(out, a, codes, scales, group, bias, epi, residual):
    w = codes.double() * scales.double().repeat_interleave(group, 1)
    y, size = a.double() @ w.t() + bias.double(), a.double().abs() @ w.abs().t() + bias.double().abs()
    K = w.shape[1]
    limit = (8 * 2.0 ** -23 + (K / group + 32) * 2.0 ** -24) * size
    if epi == 1:
        y = y + residual.double()
        limit = limit + 2.0 ** -24 * y.abs()
    elif epi == 2:
        y, limit = 0.5 * y * torch.erfc(-y / 2 ** 0.5), 1.13 * limit + 2.0 ** -20 * y.abs()
        limit = limit + HALF[out.dtype] * y.abs() + 2.0 ** -24
    else:
        limit = limit + HALF[out.dtype] * y.abs()
    err = (out.double() - y).abs()
    assert bool((err <= limit * (1 + 2.0 ** -7)).all()), "error %.3g of the bound" % float((err / limit).max())


@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("N,K,group", [(16, 64, 32), (16, 64, 64), (112, 64, 32), (768, 768, 64), (2304, 256, 128), (16, 4096, 32), (4096, 1024, 128), (9504, 192, 64)])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 17, 31, 32, 33, 70])
def test_linear(models, operand, N, K, group, M):
    m, gen = models[operand], gen_of(N + K + M)
    q = m.quantize_weights(matrix(gen, N, K), group)
    codes, scales = unpack(q)
    a = randn(gen, M, K + 16).to(TYPES[operand])
    bias = randn(gen, N)
    for epi in range(3):
        residual = randn(gen, M, N)
        guard = torch.full((M + 3, N), 7.0, device="cuda", dtype=(torch.bfloat16, torch.float32, TYPES[operand])[epi])
        if epi == 1:
            guard[:M] = residual
        m.linear_quantized(a[:, 8:8 + K], q, bias, epi, guard, M=M, lda=K + 16)
        assert_linear(guard[:M], a[:, 8:8 + K], codes, scales, group, bias, epi, residual)
        assert bool((guard[M:] == 7).all())
        if epi != 1:
            again = torch.empty(M, N, dtype=guard.dtype, device="cuda")
            m.linear_quantized(a[:, 8:8 + K], q, bias, epi, again, lda=K + 16)
            assert torch.equal(again, guard[:M])


@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("N,K,group", [(4752, 4160, 64), (4768, 4160, 32), (16384, 640, 128), (14240, 704, 32), (9600, 2112, 64), (18960, 640, 64)])
@pytest.mark.parametrize("M", [1, 8, 13, 16, 20, 31, 41])
def test_linear_of_large_matrices(models, operand, N, K, group, M):
    """Matrices that flow through a ring: ragged last units, last stages and last groups of rows."""
    m, gen = models[operand], gen_of(N + K + M)
    q = m.quantize_weights(matrix(gen, N, K), group)
    codes, scales = unpack(q)
    a, bias, residual = randn(gen, M, K).to(TYPES[operand]), randn(gen, N), randn(gen, M, N)
    out = residual.clone()
    m.linear_quantized(a, q, bias, 1, out)
    assert_linear(out, a, codes, scales, group, bias, 1, residual)
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for o in outs:
        m.linear_quantized(a, q, bias, 0, o)
    assert_linear(outs[0], a, codes, scales, group, bias, 0, None)
    assert torch.equal(*outs)


@pytest.mark.parametrize("N,K,M", [(768, 256, 2), (4768, 4160, 3), (4768, 4160, 20)])
def test_weights_laid_out_right_before_the_product(models, N, K, M):
    """A projection fetches its first codes ahead of what the kernel before it wrote, but not ahead of its own weights' layout."""
    m, gen = models["bf16"], gen_of(N + M)
    a, bias = randn(gen, M, K).to(torch.bfloat16), randn(gen, N)
    ws = [matrix(gen, N, K) * (i + 1) for i in range(4)]
    want = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in ws]
    for w, o in zip(ws, want):
        q = m.quantize_weights(w, 64)
        torch.cuda.synchronize()
        m.linear_quantized(a, q, bias, 0, o)
    out = [torch.empty_like(o) for o in want]
    for _ in range(5):
        for w, o in zip(ws, out):
            assert m.lib.marche_quantize_weights(m.h, w.data_ptr(), q.ref, torch.cuda.current_stream().cuda_stream) == 0   # (without the binding's wait)
            m.linear_quantized(a, q, bias, 0, o)
        assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_every_code_and_a_scale_that_is_not_a_number(models):
    """-8, which the quantiser does not give, is a code like the others; a NaN scale reaches its outputs only."""
    for operand in TYPES:
        m, gen = models[operand], gen_of(9)
        q = m.quantize_weights(matrix(gen, 32, 128), 64)
        q.codes.copy_(torch.randint(0, 256, q.codes.shape, generator=gen, device="cuda").to(torch.uint8))
        q.scales.copy_(torch.rand(q.scales.shape, generator=gen, device="cuda") + 0.5)
        codes, scales = unpack(q)
        assert int(codes.min()) == -8 and int(codes.max()) == 7
        a, bias, out = randn(gen, 3, 128).to(TYPES[operand]), randn(gen, 32), torch.empty(3, 32, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        m.linear_quantized(a, q, bias, 0, out)
        assert_linear(out, a, codes, scales, 64, bias, 0, None)
        q.scales[10] = float("nan")                                  # tile 0, group 0, output 5
        torch.cuda.synchronize()
        m.linear_quantized(a, q, bias, 0, out)
        assert bool(out[:, 5].isnan().all()) and int(out.isnan().sum()) == 3
        w = matrix(gen, 16, 64)
        w[2, 3], w[4, 40] = float("inf"), float("nan")
        s = unpack(m.quantize_weights(w, 32))[1]
        assert s.isnan().sum() == 2 and bool(s[2, 0].isnan()) and bool(s[4, 1].isnan())


@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("M", [5, 12, 20])
def test_every_code_of_a_large_matrix(models, operand, M):
    """The kernels for large matrices on codes -8 .. 7, a NaN scale, which reaches its output only, and an infinite value, which reaches its row only."""
    m, gen, N, K = models[operand], gen_of(M), 4768, 4160
    q = m.quantize_weights(matrix(gen, N, K), 32)
    q.codes.copy_(torch.randint(0, 256, q.codes.shape, generator=gen, device="cuda").to(torch.uint8))
    q.scales.copy_(torch.rand(q.scales.shape, generator=gen, device="cuda") + 0.5)
    codes, scales = unpack(q)
    assert int(codes.min()) == -8 and int(codes.max()) == 7
    a, bias, out = randn(gen, M, K).to(TYPES[operand]), randn(gen, N), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    m.linear_quantized(a, q, bias, 0, out)
    assert_linear(out, a, codes, scales, 32, bias, 0, None)
    q.scales[10] = float("nan")                                      # tile 0, group 0, output 5
    codes[:, 7] = 1
    q2 = a.clone()
    q2[3, 7] = float("inf")
    torch.cuda.synchronize()
    other = torch.empty_like(out)
    m.linear_quantized(q2, q, bias, 0, other)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[3], keep[:, 5] = False, False
    assert bool(other[:, 5].isnan().all()) and not bool(other[3].isfinite().all()) and torch.equal(other[keep], out[keep])


@pytest.mark.parametrize("M", [2, 12, 31])
def test_projections_on_two_streams_and_in_graphs(models, M):
    """Small and large matrices beside the attention with many rows: on two streams at once, captured on both, replayed over new inputs at once."""
    m, gen = models["f16"], gen_of(M)
    shapes = [(768, 256, 64), (4768, 4160, 64), (9600, 2112, 32)]
    ws = [m.quantize_weights(matrix(gen, N, K), g) for N, K, g in shapes]
    bias = [randn(gen, w.N) for w in ws]
    cache = filled_cache(m, gen, 20, 320, 8, 64)
    rows = [[randn(gen, M, w.K).to(torch.float16) for w in ws] for _ in range(2)]
    q = randn(gen, 20 * 70, 8 * 64).to(torch.bfloat16)

    def all_of(side, out, o):
        for a, w, b, y in zip(rows[side], ws, bias, out):
            m.linear_quantized(a, w, b, 0, y)
            m.attention_quantized(q, 512, 70, 8, cache, None, o)
            m.linear_quantized(a, w, b, 0, y)
    new = lambda: ([torch.empty(M, w.N, dtype=torch.bfloat16, device="cuda") for w in ws], torch.empty(20 * 70, 512, dtype=torch.float16, device="cuda"))
    want, got, sides = [new(), new()], [new(), new()], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        all_of(k, *want[k])
    torch.cuda.synchronize()
    same = lambda: all(torch.equal(x, y) for k in range(2) for x, y in zip(want[k][0] + [want[k][1]], got[k][0] + [got[k][1]]))
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(sides[k]):
                all_of(k, *got[k])
    torch.cuda.synchronize()
    assert same()
    for k in range(2):
        with torch.cuda.graph(graphs[k], stream=sides[k]):
            all_of(k, *got[k])
    for r in rows[0] + rows[1]:
        r.neg_()
    for k in range(2):
        all_of(k, *want[k])
    torch.cuda.synchronize()
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(sides[k]):
                graphs[k].replay()
    torch.cuda.synchronize()
    assert same()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("B,S,n", [(2, 333, 1), (2, 320, 13), (10, 100, 20)])
def test_one_block_of_a_step_in_narrow_formats(models, operand, B, S, n):
    """q, k, v by 4-bit weights; k, v of the active tokens into the 8-bit cache; attention; output projection onto the residual rows: each call
    on what the call before it left, enqueued without a wait, as a step does."""
    m, gen, H, dh, group = models[operand], gen_of(S + n), 4, 64, 64
    D = H * dh
    w_qkv, w_o = (m.quantize_weights(randn(gen, N, D) * D ** -0.5, group) for N in (3 * D, D))
    cache = filled_cache(m, gen, B, S, H, dh)
    u = randn(gen, B * n, D).to(TYPES[operand])
    b_qkv, b_o, x = randn(gen, 3 * D), randn(gen, D), randn(gen, B * n, D)
    residual = x.clone()
    idx = torch.rand(B, S, generator=gen, device="cuda").argsort(1)[:, :n].to(torch.int32).contiguous()
    qkv = torch.empty(B * n, 3 * D, dtype=torch.bfloat16, device="cuda")
    o = torch.empty(B * n, D, dtype=TYPES[operand], device="cuda")
    m.linear_quantized(u, w_qkv, b_qkv, binding.EPI_BIAS, qkv)
    m.scatter_kv_quantized(qkv[:, D:2 * D], qkv[:, 2 * D:], 3 * D, idx, n, cache)
    m.attention_quantized(qkv, 3 * D, n, H, cache, None, o)
    m.linear_quantized(o, w_o, b_o, binding.EPI_BIAS_RESIDUAL, x)
    torch.cuda.synchronize()
    codes, scales = unpack(w_qkv)
    assert_linear(qkv, u, codes, scales, group, b_qkv, 0, None)
    c, _ = definition(torch.stack([qkv[:, D:2 * D], qkv[:, 2 * D:]]).view(2, B, n, H, dh))
    got = torch.gather(cache.codes, 2, idx.long().view(1, B, n, 1).expand(2, B, n, D))
    assert torch.equal(got.view_as(c), c.to(torch.int8))
    assert_attention(o, cache, qkv[:, :D], n, H, None)
    codes, scales = unpack(w_o)
    assert_linear(x, o, codes, scales, group, b_o, 1, residual)


# ------------------------------------------------------------------ refusals
def test_refusals(models):
    """Refused on the host: nothing is enqueued, the launch count stays."""
    m, f32 = models["f16"], make_model(synth.CONFIGS["tiny"], synth.make_weights(synth.CONFIGS["tiny"]))
    B, S, H, dh, n = 2, 64, 2, 64, 4
    D = H * dh
    cache, rows = m.alloc_quantized_cache(B, S, H, dh), torch.zeros(B * n, D + 8, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(B * n, D + 8, dtype=torch.float16, device="cuda")
    w = m.quantize_weights(torch.zeros(32, 128, device="cuda"), 64)
    bias = torch.zeros(32, device="cuda")
    lib, h, p, r, oo = m.lib, m.h, rows.data_ptr(), cache.ref, out.data_ptr()
    before = m.launch_count()

    def shaped(**kw):
        c = binding.MarcheQuantizedCache(cache.codes.data_ptr(), cache.scales.data_ptr(), B, S, H, dh)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    def attention(q=p, ld=D + 8, rows_=n, heads=H, c=None, ctx=h, o=oo):
        return lib.marche_attention_quantized(ctx, q, ld, rows_, heads, r if c is None else binding.C.addressof(c), None, o, None)

    EINVAL, ESHAPE = -1, -2
    assert attention(ctx=f32.h) == ESHAPE
    assert attention(q=p + 2) == EINVAL and attention(ld=D + 4) == EINVAL and attention(ld=D - 8) == EINVAL
    assert attention(rows_=-1) == EINVAL and attention(heads=3) == EINVAL and attention(heads=0) == EINVAL and attention(o=oo + 4) == EINVAL
    assert attention(rows_=0) == 0
    for kw, code in [(dict(head_dim=72), ESHAPE), (dict(head_dim=32), ESHAPE), (dict(batch=0), EINVAL), (dict(seq_len=0), EINVAL), (dict(n_kv_heads=0), EINVAL),
                     (dict(codes=0), EINVAL), (dict(scales=0), EINVAL), (dict(seq_len=(1 << 24) + 1), ESHAPE), (dict(codes=cache.codes.data_ptr() + 8), EINVAL),
                     (dict(batch=1 << 30), ESHAPE)]:
        assert attention(c=shaped(**kw)) == code, kw
    assert attention(rows_=1 << 25, ld=D + 8) == ESHAPE

    def scatter(k=p, ld=D + 8, idx=None, rows_=n, ctx=h):
        return lib.marche_scatter_kv_quantized(ctx, k, p, ld, idx, rows_, r, None)

    def gather(k=p, ld=D + 8, idx=None, rows_=n, ctx=h):
        return lib.marche_gather_kv_quantized(ctx, r, idx, rows_, k, p, ld, None)

    for call in (scatter, gather):
        assert call(ctx=f32.h) == ESHAPE and call(k=None) == EINVAL and call(k=p + 8) == EINVAL and call(ld=D + 4) == EINVAL
        assert call(ld=D - 8) == EINVAL and call(rows_=S + 1) == EINVAL and call(rows_=-1) == EINVAL and call(rows_=0) == 0
        assert call(rows_=1 << 30, idx=p) == ESHAPE

    def linear(a=p, lda=136, M=4, epi=0, o=oo, ctx=h, **kw):
        c = binding.MarcheQuantizedWeights(w.codes.data_ptr(), w.scales.data_ptr(), 32, 128, 64)
        for k, v in kw.items():
            setattr(c, k, v)
        return lib.marche_linear_quantized(ctx, a, lda, M, binding.C.addressof(c), bias.data_ptr(), epi, o, None)

    assert linear(ctx=f32.h) == ESHAPE and linear(group=16) == ESHAPE and linear(n=24) == ESHAPE and linear(k=96) == ESHAPE and linear(M=65537) == ESHAPE
    assert linear(a=None) == EINVAL and linear(lda=120) == EINVAL and linear(lda=132) == EINVAL and linear(epi=3) == EINVAL and linear(M=-1) == EINVAL
    assert linear(codes=0) == EINVAL and linear(a=p + 2) == EINVAL and linear(o=oo + 2) == EINVAL and linear(M=0) == 0
    assert m.launch_count() == before
    with pytest.raises(MarcheError):
        m.alloc_quantized_cache(1, 1, 1, 96)
    with pytest.raises(MarcheError):
        m.quantize_weights(torch.zeros(24, 64, device="cuda"), 64)
    with pytest.raises(AssertionError):                              # fewer rows than the call names
        m.scatter_kv_quantized(rows, rows, D + 8, None, n + 1, cache)
    with pytest.raises(AssertionError):
        m.attention_quantized(rows, D + 8, n, H, cache, torch.zeros(1, dtype=torch.int32, device="cuda"), out)
    with pytest.raises(AssertionError):
        QuantizedCache(cache.codes, cache.scales[..., :32].contiguous(), H)


# ------------------------------------------------------------------ rows, keys and sizes that have nothing to do with one another
@pytest.mark.parametrize("dh,heads,kv_heads", [(64, 2, 2), (64, 8, 2), (80, 3, 3), (128, 4, 2)])
@pytest.mark.parametrize("n", [1, 3, 20, 140])
@pytest.mark.parametrize("operand", ["f16", "bf16"])
def test_a_query_row_does_not_reach_other_rows(models, both_kernels, operand, dh, heads, kv_heads, n):
    """Rows of padding may hold any finite numbers: the rows beside them keep their results, bit for bit."""
    m, gen, B, S = models[operand], gen_of(n + dh + heads), 3, 333
    cache = filled_cache(m, gen, B, S, kv_heads, dh)
    q = randn(gen, B * n, heads, dh).to(torch.bfloat16)
    want = attend(m, cache, q.view(B * n, -1), heads * dh, n, heads, None).view(B * n, heads, dh)
    assert_attention(want, cache, q.view(B * n, -1), n, heads, None)
    for power, at in [(33, -1), (60, 0), (120, n // 2), (60, 2 * n - 1)]:
        other = q.clone()
        if power == 60:
            other[at, heads - 1] *= 2.0 ** power                     # one row of one head
        else:
            other[at, heads // 2, 5] = -3 * 2.0 ** power             # one value of it
        o = attend(m, cache, other.view(B * n, -1), heads * dh, n, heads, None).view(B * n, heads, dh)
        same_row = (other == q).all(-1)
        assert int((~same_row).sum()) == 1
        assert torch.equal(o[same_row], want[same_row]), (power, at)
        assert bool(o.isfinite().all())


@pytest.mark.parametrize("n", [2, 40, 140])
def test_rows_of_all_sizes_side_by_side(models, both_kernels, n):
    """Rows from 2^-100 to 2^6, a power of two apart, and rows whose own values are 2^45 apart."""
    m, gen, B, S, H, dh = models["f16"], gen_of(n), 2, 200, 3, 64
    cache = filled_cache(m, gen, B, S, H, dh)
    q = randn(gen, B * n, H, dh) * torch.exp2(torch.randint(-100, 7, (B * n, H, 1), generator=gen, device="cuda").float() * (torch.rand(B * n, H, 1, generator=gen, device="cuda") < 0.7))
    q[::3, :, ::2] *= 2.0 ** -45
    q = (q / q.abs().amax(-1, keepdim=True).clamp_min(6.0) * 6.0).to(torch.bfloat16).view(B * n, H * dh)
    assert_attention(attend(m, cache, q, H * dh, n, H, None), cache, q, n, H, None)


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("n,S", [(1, 9), (20, 9), (20, 150), (140, 150)])
def test_rows_of_one_sign_over_small_codes(models, both_kernels, dh, n, S):
    """One channel of K is large, so that the others' codes are small, and no row has anything there: a logit is a sum of small products, and only
    they may round.  8 steps of the tensor cores at most, 2^-23 of the sum of magnitudes each, and three roundings of 2^-24: 2^-19.5 of it; a
    weight is off by that share of itself, once for its own logit and once for the sum's."""
    m, gen, B, H = models["f16"], gen_of(n), 12, 4
    x = randn(gen, 2, B, S, H, dh)
    x[0, ..., 3] = 100 * (1 + torch.rand(B, S, H, generator=gen, device="cuda"))
    c, s = definition(x.to(torch.bfloat16))
    cache = m.alloc_quantized_cache(B, S, H, dh)
    cache.codes.copy_(c.to(torch.int8).view_as(cache.codes))
    cache.scales[..., :S] = s.transpose(2, 3)
    q = 6 * randn(gen, B * n, H, dh).abs()
    q[..., 3] = 0
    q = q.to(torch.bfloat16).view(B * n, H * dh)
    o = attend(m, cache, q, H * dh, n, H, None).double().view(B * n, H, dh)
    want, A, low = reference(cache, q, n, H, None)
    size = torch.einsum("bnhd,bshd->bnhs", q.double().view(B, n, H, dh), values(cache)[0].abs()).amax(-1).view(B * n, H, 1) / dh ** 0.5
    rounding = 2.0 ** -11 if both_kernels == "tcgen05" else 2.0 ** -22        # of the weights
    limit = (rounding + 2 * 2.0 ** -19.5 * size) * A + low + HALF[torch.float16] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -24
    assert bool(((o - want).abs() <= limit).all()), "error %.3g of the bound" % float(((o - want).abs() / limit).max())


def test_keys_at_the_upper_end_of_the_range(models, both_kernels):
    """K near the largest bf16 number and rows near the smallest: the logits are ordinary."""
    m, gen, B, S, H, dh = models["bf16"], gen_of(12), 1, 200, 2, 64
    cache = filled_cache(m, gen, B, S, H, dh, spread=False)
    cache.scales[0] *= 2.0 ** 124                                     # up to 2^120 a code
    assert float(cache.scales[0, :, :, :S].max()) > 2.0 ** 119 and bool((127 * cache.scales[0, :, :, :S]).isfinite().all())
    for n in (3, 140):
        q = (randn(gen, B * n, H * dh) * 2.0 ** -121).to(torch.bfloat16)
        assert_attention(attend(m, cache, q, H * dh, n, H, None), cache, q, n, H, None)


def outlier_reference(cache, q, n, heads, kv_len):
    """o, A and S 127 max(p vs) of the row itself: what its smallest steps are relative to."""
    o, A, _ = reference(cache, q, n, heads, kv_len)
    B, S, Hkv, dh = cache.B, cache.S, cache.n_kv_heads, cache.head_dim
    k, vs = values(cache)[0], cache.scales[1, :, :, :S].double()
    x = torch.einsum("bnhd,bshd->bnhs", q.double().view(B, n, heads, dh), k.repeat_interleave(heads // Hkv, 2)) / dh ** 0.5
    if kv_len is not None:
        x = x.masked_fill(torch.arange(S, device="cuda") >= kv_len.view(B, 1, 1, 1), float("-inf"))
    p = torch.softmax(x, -1).nan_to_num(0.0)
    top = (p * vs.repeat_interleave(heads // Hkv, 1).unsqueeze(1).nan_to_num(0.0)).amax(-1)
    return o, A, (S * 127 * top).view(B * n, heads, 1)


@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("dh,heads,kv_heads,n", [(64, 2, 2, 1), (64, 4, 1, 30), (80, 2, 2, 140), (128, 2, 2, 20), (128, 4, 4, 150)])
@pytest.mark.parametrize("power,logit", [(20, -25.0), (45, -25.0), (60, -60.0), (100, -60.0), (119, -200.0), (-60, 30.0)])
@pytest.mark.parametrize("where", ["first", "middle", "last", "tile", "all but few"])
def test_a_value_without_weight_does_not_push_the_others_out(models, both_kernels, where, power, logit, dh, heads, kv_heads, n, operand):
    """Keys whose value scale lies far above (below) the others' at a weight of next to nothing (of nearly all).  A weight is off by half a step of
    2^-24 at most, and the row's largest product of weight and value scale is kept at 2^-4 or above: S 2^-21 127 max(p vs) bounds what
    the steps of small weights do; else the bounds of all tests here."""
    m, gen, B, S = models[operand], gen_of(n + dh), 2, 700
    cache = filled_cache(m, gen, B, S, kv_heads, dh, spread=False)
    keys = {"first": slice(0, 1), "middle": slice(330, 332), "last": slice(S - 1, S), "tile": slice(0, 64), "all but few": slice(5, 690)}[where]
    ones = cache.codes[0].view(B, S, kv_heads, dh)
    ones[:, keys] = 0
    ones[:, keys, :, 0] = 127 if logit > 0 else -127                 # k = -+ that, 0, 0, ..: q's first value is 8
    cache.scales[0, :, :, keys] = abs(logit) * dh ** 0.5 / 8 / 127
    cache.scales[1, :, :, keys] *= 2.0 ** power
    if where != "all but few":
        cache.scales[1, 1, :, keys] *= 2.0 ** -7                      # (samples differ)
    q = randn(gen, B * n, heads, dh)
    q[:, :, 0] = 8
    q = q.to(torch.bfloat16).view(B * n, heads * dh)
    for kv_len in (None, torch.tensor([S - 3, 340], dtype=torch.int32, device="cuda")):
        o = attend(m, cache, q, heads * dh, n, heads, kv_len)
        want, A, low = outlier_reference(cache, q, n, heads, kv_len)
        # sums of |q k| reach 2^11 beside the keys of the given logit: off by 2^11 2^-22 sqrt(1 / dh); a value beyond the type's end is not asked for
        limit = (2.0 ** -11 + 2.0 ** -10) * A + 2.0 ** -21 * low + HALF[o.dtype] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -24
        fits = want.abs() < 6e4
        assert bool(((o.double().view_as(want) - want).abs() <= limit)[fits].all())
        assert torch.equal(o, attend(m, cache, q, heads * dh, n, heads, kv_len)) or not bool(fits.all())


def test_values_far_apart_in_some_samples_only(models, both_kernels):
    """More units than SMs: what a unit met does not follow into the next one."""
    m, gen, B, S, H, dh, n = models["f16"], gen_of(8), 120, 200, 4, 64, 150
    cache = filled_cache(m, gen, B, S, H, dh)
    q = randn(gen, B * n, H * dh).to(torch.bfloat16)
    want = attend(m, cache, q, H * dh, n, H, None)
    cache.scales[1, ::3, 1, 7] *= 2.0 ** 60
    cache.scales[1, 1::3, :, 100:] *= 2.0 ** -50
    o = attend(m, cache, q, H * dh, n, H, None).view(B, n, H, dh)
    assert torch.equal(o[2::3], want.view_as(o)[2::3]) and torch.equal(o[::3, :, [0, 2, 3]], want.view_as(o)[::3, :, [0, 2, 3]])
    for b in (1, 4, 58, 118):
        part = QuantizedCache(cache.codes[:, b:b + 1].contiguous(), cache.scales[:, b:b + 1].contiguous(), H)
        assert_attention(o[b], part, q[b * n:(b + 1) * n], n, H, None)


def test_rows_with_infinities_beside_ordinary_ones(models, both_kernels):
    """A row that holds an infinity or a NaN has no numbers in its result; the rows beside it keep theirs."""
    m, gen, B, S, H, dh, n = models["f16"], gen_of(15), 2, 150, 2, 80, 37
    cache = filled_cache(m, gen, B, S, H, dh)
    q = randn(gen, B * n, H, dh).to(torch.bfloat16)
    want = attend(m, cache, q.view(B * n, -1), H * dh, n, H, None).view(B * n, H, dh)
    bad = q.clone()
    bad[3, 0, 7], bad[5, 1, 79], bad[40, 1, 0], bad[40, 1, 1] = float("inf"), float("nan"), float("-inf"), 1e30
    o = attend(m, cache, bad.view(B * n, -1), H * dh, n, H, None).view(B * n, H, dh)
    rest = torch.ones(B * n, H, dtype=torch.bool, device="cuda")
    for row, head in ((3, 0), (5, 1), (40, 1)):
        assert bool(o[row, head].isnan().all())
        rest[row, head] = False
    assert torch.equal(o[rest], want[rest])


def test_no_rows_at_all(models):
    """A call without rows enqueues nothing, whatever its empty tensors point to."""
    m = models["f16"]
    cache, w = m.alloc_quantized_cache(2, 64, 2, 64), m.quantize_weights(torch.zeros(32, 128, device="cuda"), 64)
    bf, f16 = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 128, dtype=torch.float16, device="cuda")
    before = m.launch_count()
    m.scatter_kv_quantized(bf, bf, 128, None, 0, cache)
    m.scatter_kv_quantized(bf, bf, 128, torch.empty(2, 0, dtype=torch.int32, device="cuda"), 0, cache)
    m.gather_kv_quantized(cache, None, 0, bf, bf, 128)
    m.attention_quantized(bf, 128, 0, 2, cache, None, f16)
    for epi, dtype in enumerate((torch.bfloat16, torch.float32, torch.float16)):
        m.linear_quantized(f16, w, torch.zeros(32, device="cuda"), epi, torch.empty(0, 32, dtype=dtype, device="cuda"))
    assert m.launch_count() == before


def test_rows_as_tensors_come(models):
    """One row has no stride; rows whose values do not lie side by side are refused."""
    m, gen, N, K = models["f16"], gen_of(13), 32, 128
    w = m.quantize_weights(matrix(gen, N, K), 64)
    codes, scales = unpack(w)
    a, bias, out = randn(gen, K, 1).to(torch.float16).t(), randn(gen, N), torch.empty(1, N, dtype=torch.bfloat16, device="cuda")
    assert a.stride(0) < K
    for kw in ({}, dict(M=1)):
        out.zero_()
        m.linear_quantized(a, w, bias, 0, out, **kw)
        assert_linear(out, a, codes, scales, 64, bias, 0, None)
    wide, out = randn(gen, 4, 2 * K).to(torch.float16), torch.empty(4, N, dtype=torch.bfloat16, device="cuda")
    for kw in ({}, dict(M=4), dict(M=4, lda=2 * K)):
        with pytest.raises(AssertionError):
            m.linear_quantized(wide[:, ::2], w, bias, 0, out, **kw)
    cache, rows, o = m.alloc_quantized_cache(1, 64, 2, 64), torch.zeros(4, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 128, dtype=torch.float16, device="cuda")
    with pytest.raises(AssertionError):
        m.scatter_kv_quantized(rows[:, ::2], rows[:, ::2], 512, None, 4, cache)
    with pytest.raises(AssertionError):
        m.gather_kv_quantized(cache, None, 4, rows[:, ::2], rows[:, ::2], 512)
    with pytest.raises(AssertionError):
        m.attention_quantized(rows[:, ::2], 512, 4, 2, cache, None, o)



def test_weights_laid_out_on_another_stream(models):
    """Memory that the current stream gave back, but has not finished with, may be what the layout gets."""
    m, gen, N, K = models["f16"], gen_of(14), 4096, 8192
    w = matrix(gen, N, K)
    want = m.quantize_weights(w, 64)
    codes, scales = want.codes.clone(), want.scales.clone()
    side = torch.cuda.Stream()
    del want
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    left = [torch.empty(N * K // 2, dtype=torch.uint8, device="cuda") for _ in range(4)]
    at = {t.data_ptr() for t in left}
    left += [torch.empty(N * K // 64, dtype=torch.bfloat16, device="cuda").view(torch.uint8) for _ in range(4)]   # (nothing is to be allocated anew)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for t in left:
        t.fill_(255)
    del left, t
    got = m.quantize_weights(w, 64, stream=side)
    torch.cuda.synchronize()
    assert got.codes.data_ptr() in at
    assert torch.equal(got.codes, codes) and torch.equal(got.scales, scales)


@pytest.mark.parametrize("dh,n", [(64, 1), (80, 30), (128, 3), (64, 140), (128, 150)])
@pytest.mark.parametrize("power", [0, 40])
def test_scales_of_either_sign_and_every_code(models, both_kernels, dh, n, power):
    """A cache that others have filled: scales below 0, codes of -128; some value scales far below the rest."""
    m, gen, B, S, H = models["f16"], gen_of(n + dh), 2, 300, 2
    cache = filled_cache(m, gen, B, S, H, dh)
    cache.codes.copy_(torch.randint(-128, 128, cache.codes.shape, generator=gen, device="cuda").to(torch.int8))
    assert int(cache.codes.min()) == -128
    cache.scales *= torch.where(torch.rand(cache.scales.shape, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    cache.scales[1, 0, :, 7] *= 2.0 ** -power
    q = (0.3 * randn(gen, B * n, H * dh)).to(torch.bfloat16)
    assert_attention(attend(m, cache, q, H * dh, n, H, None), cache, q, n, H, None)


@pytest.mark.parametrize("dh,n", [(64, 1), (80, 30), (128, 3), (64, 140), (128, 150)])
def test_values_at_the_upper_end_of_the_range(models, both_kernels, dh, n):
    """V near the largest bf16 number: the mean is one, though the sum over the keys would not be."""
    m, gen, B, S, H = models["bf16"], gen_of(n + dh), 2, 1500, 2
    cache = filled_cache(m, gen, B, S, H, dh, spread=False)
    q = randn(gen, B * n, H * dh).to(torch.bfloat16)
    cache.scales[1] /= 127 * cache.scales[1, :, :, :S].max()
    cache.scales[1] *= 2.0 ** 127                                     # (codes of 127 are 2^127)
    o = attend(m, cache, q, H * dh, n, H, None)
    want, A, low = reference(cache, q, n, H, None)
    limit = (2.0 ** -11 + 2.0 ** -13) * A + low + HALF[o.dtype] * want.abs() * (1 + 2.0 ** -10)
    assert bool(((o.double().view_as(want) - want).abs() <= limit).all())


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("n,S", [(3, 2), (5, 2), (16, 5), (1, 40)])
def test_what_the_weights_rounding_left_off(models, dh, n, S):
    """fp16 outputs of the mma.sync kernel: the rest of a weight is a second operand.  Values that cancel, so that the output's own rounding hides
    nothing: what is left are logits of |x| < 2^4 (2^-18 of them: 2^-17.5 of a weight with the sum's) and 2^-21 of the weights."""
    m, gen, B, H = models["f16"], gen_of(n + S + dh), 8, 4
    m.set_tuning(attention_kernel=KERNELS["mma"])
    try:
        cache = filled_cache(m, gen, B, S, H, dh, spread=False)
        q = (0.5 * randn(gen, B * n, H * dh)).to(torch.bfloat16)
        p = torch.softmax(torch.einsum("bnhd,bshd->bnhs", q.double().view(B, n, H, dh), values(cache)[0]) / dh ** 0.5, -1)
        # the second key's values cancel the first one's for the first token's weights, nearly
        cache.codes[1, :, 0] = 127
        cache.codes[1, :, 1] = -127
        cache.scales[1, :, :, 0], cache.scales[1, :, :, 1] = p[:, 0, :, 1].float(), p[:, 0, :, 0].float()
        o = attend(m, cache, q, H * dh, n, H, None).double().view(B * n, H, dh)
        want, A, low = reference(cache, q, n, H, None)
        limit = (2.0 ** -21 + 2.0 ** -17.5) * A + low + HALF[torch.float16] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -25
        assert bool(((o - want).abs() <= limit).all()), "error %.3g of the bound" % float(((o - want).abs() / limit).max())
    finally:
        m.set_tuning(attention_kernel=binding.ATTENTION_AUTO)


# ------------------------------------------------------------------ large matrices, all forms
LARGE = [  # N, K, group: every kernel for large matrices at every group, pairs with one unit and with several in turn, a single stage of one chunk among them
    (4864, 4224, 128), (4864, 4224, 64), (4864, 4224, 32), (12288, 2304, 128), (12288, 2304, 64), (12288, 2304, 32), (24576, 1152, 128), (24576, 1152, 64), (24576, 1152, 32),
    (16384, 1024, 128), (18960, 640, 64), (18960, 640, 32), (151568, 64, 32), (151568, 64, 64), (75792, 128, 128)]
LARGE_ROWS = [1, 5, 8, 9, 16, 17, 29, 32, 45]


@pytest.fixture(scope="module")
def large_matrix(models):
    """(N, K, group) -> the matrix laid out, its codes and scales; the last one is kept, since the tests below take them in turn."""
    last = {}

    def get(N, K, group):
        if (N, K, group) not in last:
            last.clear()
            q = models["f16"].quantize_weights(matrix(gen_of(N + K), N, K), group)
            last[N, K, group] = (q,) + unpack(q)
        return last[N, K, group]
    return get


@pytest.mark.parametrize("operand", ["f16", "bf16"])
@pytest.mark.parametrize("M", LARGE_ROWS)
@pytest.mark.parametrize("N,K,group", LARGE)
def test_linear_of_large_matrices_with_all_epilogues(models, large_matrix, operand, N, K, group, M):
    m, gen = models[operand], gen_of(N + K + M)
    q, codes, scales = large_matrix(N, K, group)
    a, bias = randn(gen, M, K + 24).to(TYPES[operand])[:, 8:8 + K], randn(gen, N)
    for epi in range(3):
        residual = randn(gen, M, N)
        out = torch.full((M + 2, N), 7.0, device="cuda", dtype=(torch.bfloat16, torch.float32, TYPES[operand])[epi])
        if epi == 1:
            out[:M] = residual
        m.linear_quantized(a, q, bias, epi, out, M=M, lda=K + 24)
        assert_linear(out[:M], a, codes, scales, group, bias, epi, residual)
        assert bool((out[M:] == 7).all())


@pytest.mark.parametrize("N,K,group,M", [(768, 768, 64, 1088), (4864, 4224, 128, 500), (2304, 768, 32, 1000), (64, 128, 64, 65536), (9600, 2112, 64, 161)])
def test_linear_of_many_rows(models, N, K, group, M):
    m, gen = models["f16"], gen_of(N + M)
    q = m.quantize_weights(matrix(gen, N, K), group)
    codes, scales = unpack(q)
    a, bias, out = randn(gen, M, K).to(torch.float16), randn(gen, N), torch.empty(M, N, dtype=torch.float16, device="cuda")
    m.linear_quantized(a, q, bias, 2, out)
    assert_linear(out, a, codes, scales, group, bias, 2, None)
