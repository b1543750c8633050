"""Sizes and layouts of the 8-bit cache and the 4-bit weights as the library answers them, and what it refuses before it looks at a
device (no GPU needed)."""
import ctypes as C

import pytest

ESHAPE, EINVAL = -2, -1


@pytest.fixture(scope="module")
def lib():
    from paper_2506_12035_b200 import binding, build
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("B,S,H,dh", [(1, 1, 1, 64), (2, 64, 12, 64), (3, 65, 16, 80), (128, 320, 16, 128), (2, 1 << 20, 8, 128)])
def test_cache_sizes(lib, B, S, H, dh):
    assert lib.marche_quantized_codes_bytes(B, S, H, dh) == 2 * B * S * H * dh
    assert lib.marche_quantized_scales_bytes(B, S, H, dh) == 2 * B * H * ((S + 63) // 64 * 64) * 4


@pytest.mark.parametrize("B,S,H,dh", [(0, 1, 1, 64), (1, 0, 1, 64), (1, 1, 0, 64), (1, 1, 1, 48), (1, 1, 1, 96), (-1, 1, 1, 64)])
def test_cache_sizes_of_what_is_not_supported(lib, B, S, H, dh):
    assert lib.marche_quantized_codes_bytes(B, S, H, dh) == 0 and lib.marche_quantized_scales_bytes(B, S, H, dh) == 0


@pytest.mark.parametrize("n,k,group,ok", [(16, 64, 32, True), (16, 64, 64, True), (16, 64, 128, False), (768, 768, 128, True), (48, 192, 64, True),
                                          (48, 192, 128, False), (8, 64, 64, False), (24, 64, 64, False), (16, 96, 32, False),
                                          (16, 64, 16, False), (0, 64, 64, False), (16, 0, 64, False), (-16, 64, 64, False)])
def test_weight_sizes(lib, n, k, group, ok):
    scales = C.c_size_t(77)
    got = lib.marche_quantized_weights_bytes(n, k, group, C.byref(scales))
    assert got == (n * k // 2 if ok else 0) and scales.value == (n * (k // group) * 2 if ok else 0)
    assert lib.marche_quantized_weights_bytes(n, k, group, None) == got


def test_null_arguments(lib):
    from paper_2506_12035_b200 import binding
    cache, w = binding.MarcheQuantizedCache(), binding.MarcheQuantizedWeights()
    p = 0x1000
    assert lib.marche_scatter_kv_quantized(None, p, p, 64, None, 1, C.addressof(cache), None) == EINVAL
    assert lib.marche_gather_kv_quantized(None, C.addressof(cache), None, 1, p, p, 64, None) == EINVAL
    assert lib.marche_attention_quantized(None, p, 64, 1, 1, C.addressof(cache), None, p, None) == EINVAL
    assert lib.marche_quantize_weights(None, p, C.addressof(w), None) == EINVAL
    assert lib.marche_linear_quantized(None, p, 64, 1, C.addressof(w), p, 0, p, None) == EINVAL
    assert C.sizeof(cache) == 32 and C.sizeof(w) == 32


class Split(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("nb", "nr", "nk", "nst", "cs", "n_rb")]


def test_attention_cuts_fit_an_sm_and_cover_all_rows(lib):
    """Every way in which a launch is cut keeps to the shared memory, the barriers and the warps of a CTA, and covers the rows."""
    plan, smem = lib._ZN6marche24attention_quantized_planEiiii, lib._ZN6marche24attention_quantized_smemEiRKNS_14QuantizedSplitE
    plan.restype, plan.argtypes = Split, [C.c_int] * 4
    smem.restype, smem.argtypes = C.c_size_t, [C.c_int, C.POINTER(Split)]
    rows = list(range(1, 34)) + [48, 49, 64, 65, 80, 96, 97, 127, 128, 129, 160, 256, 257, 300, 1000, 5000, 1 << 20]
    for dh in (64, 80, 128):
        for R in rows:
            for S in (1, 2, 63, 64, 65, 128, 129, 192, 200, 256, 257, 320, 321, 512, 576, 700, 1088, 2048, 5000, 65521, 1 << 24):
                for items in (1, 2, 8, 12, 24, 32, 60, 74, 75, 148, 149, 300, 592, 900, 2048):
                    s = plan(R, S, dh, items)
                    at = (dh, R, S, items, [getattr(s, n) for n, _ in Split._fields_])
                    assert s.nb in (1, 2) and s.nr >= 1 and s.nk >= 1 and s.nst >= 1 and s.cs in (1, 2, 4, 8), at
                    assert s.nr * s.nk <= 8 and s.nk * s.nst <= 16 and smem(dh, C.byref(s)) <= 226 * 1024, at
                    assert s.n_rb * s.nr * 8 * s.nb >= R and (s.n_rb - 1) * s.nr * 8 * s.nb < R, at
                    tiles = -(-S // (32 if dh == 128 else 64))
                    mine = -(-(-(-tiles // s.cs)) // s.nk)
                    assert s.nst >= min(mine, 3 if s.nr > 1 else 2), at            # a stage is filled again one tile late


class GemmShape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("warps", "wn", "nst", "tc")]


def test_projection_cuts_fit_an_sm(lib):
    pick, smem = lib._ZN6marche19gemm_quantized_pickEiiii, lib._ZN6marche19gemm_quantized_smemEiiRKNS_18QuantizedGemmShapeE
    pick.restype, pick.argtypes = GemmShape, [C.c_int] * 4
    smem.restype, smem.argtypes = C.c_size_t, [C.c_int, C.c_int, C.POINTER(GemmShape)]
    seen = set()
    for M in (1, 8, 9, 16, 17, 24, 25, 32, 33, 100, 65536):
        for tiles in (1, 8, 48, 144, 148, 149, 256, 296, 300, 592, 600, 888, 1024, 1536, 4096):
            for chunks in (1, 2, 3, 7, 8, 9, 12, 16, 17, 40, 64, 100, 127, 128, 129, 192, 1024):
                for group in (32, 64, 128):
                    if group == 128 and chunks % 2:
                        continue
                    s = pick(M, 16 * tiles, 64 * chunks, group)
                    at = (M, tiles, chunks, group, [getattr(s, n) for n, _ in GemmShape._fields_])
                    assert (s.warps > 0) + (s.wn > 0) + (s.tc > 0) == 1, at
                    seen.add((s.warps > 0, s.wn > 0, s.tc))
                    if s.tc:
                        assert M > 8 and s.tc in (1, 2) and (s.tc == 1 or chunks > 4), at           # a pair's halves of K are not empty
                    elif s.wn:
                        assert M <= 8 and 4 <= s.wn <= 7 and 3 <= s.nst <= 16 and smem(M, group, C.byref(s)) <= 220 * 1024, at
                    else:
                        assert s.warps <= 16 and smem(M, group, C.byref(s)) <= 48 * 1024, at
    assert seen == {(True, False, 0), (False, True, 0), (False, False, 1), (False, False, 2)}


@pytest.mark.parametrize("R,S,dh,items,want", [
    (1, 1 << 20, 64, 4096, False), (16, 320, 64, 2048, False), (43, 320, 64, 2048, False), (64, 320, 64, 2048, True), (43, 1088, 64, 512, True),
    (43, 1088, 64, 128, False), (64, 1088, 64, 128, True), (128, 1088, 64, 32, False), (200, 5000, 64, 24, False), (43, 320, 80, 2048, False),
    (1088, 1088, 64, 512, True), (32, 1088, 128, 512, False), (64, 1088, 128, 512, True)])
def test_which_attention(lib, R, S, dh, items, want):
    wins = lib._ZN6marche27attention_quantized_tc_winsEiiii
    wins.restype = C.c_bool
    assert wins(R, S, dh, items) is want


class SplitK(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("bn", "cs")]


def test_pairs_that_hold_tensor_memory_share_no_sm_with_other_clusters(lib):
    """A pair of the projections waits for its partner with all of its SM's tensor memory.  Clusters of another stream that hold some while they wait
    would, beside it, each wait for the other for good: together they need more shared memory than an SM has (228 KB, 1 KB of it for each CTA)."""
    pair, other = lib._ZN6marche22gemm_quantized_tc_smemEiii, lib._ZN6marche16gemm_splitk_smemEiiNS_11SplitKShapeE
    pair.restype, pair.argtypes = C.c_size_t, [C.c_int] * 3
    other.restype, other.argtypes = C.c_size_t, [C.c_int, C.c_int, SplitK]
    least = min(other(M, 64 * chunks, SplitK(bn, cs)) for bn, cs in [(64, 2), (64, 4), (64, 8), (32, 2), (32, 4), (128, 2), (128, 4), (128, 8)]
                for M in (1, 8, 9, 16, 100, 128, 129, 1000) for chunks in (cs, cs + 1, 12, 100) if chunks >= cs)
    for M in (9, 16, 17, 32, 33, 65536):
        for group in (32, 64, 128):
            assert pair(M, group, 1) <= pair(M, group, 2) <= 227 * 1024, (M, group)
            assert pair(M, group, 2) + 1024 + least + 1024 > 228 * 1024, (M, group)


@pytest.mark.parametrize("B,S,H,dh", [(1, (1 << 24) + 1, 1, 64), (1, 2 ** 31 - 1, 1, 64), (2, 2 ** 31 - 40, 16, 128), (1 << 24, 1, 1, 64), (1 << 20, 64, 16, 64),
                                      (2 ** 31 - 1, 1, 2 ** 31 - 1, 128)])
def test_caches_that_every_call_refuses_have_no_size(lib, B, S, H, dh):
    from paper_2506_12035_b200 import binding
    assert lib.marche_quantized_codes_bytes(B, S, H, dh) == 0 and lib.marche_quantized_scales_bytes(B, S, H, dh) == 0
    with pytest.raises(binding.MarcheError):                         # before anything is allocated
        binding.Marche.alloc_quantized_cache(type("M", (), {"lib": lib}), B, S, H, dh)


def test_largest_caches_have_a_size(lib):
    assert lib.marche_quantized_scales_bytes(1, 1 << 24, 1, 64) == 8 << 24
    assert lib.marche_quantized_codes_bytes((1 << 24) - 1, 1, 1, 64) == 128 * ((1 << 24) - 1)


@pytest.mark.parametrize("k,ok", [(64 * 65535, True), (64 * 65536, False), (2 ** 31 - 64, False)])
def test_matrices_that_cannot_be_laid_out_have_no_size(lib, k, ok):
    assert (lib.marche_quantized_weights_bytes(16, k, 64, None) == 8 * k) is ok and (lib.marche_quantized_weights_bytes(16, k, 64, None) == 0) is not ok


def test_large_matrices_of_the_gpu_tests_reach_every_kernel(lib):
    """Every kernel for large matrices that a projection can get, by rows and group, pairs with more units than there are pairs among them."""
    from test_gpu_quantized import LARGE, LARGE_ROWS
    pick = lib._ZN6marche19gemm_quantized_pickEiiii
    pick.restype, pick.argtypes = GemmShape, [C.c_int] * 4
    seen = set()
    for N, K, group in LARGE:
        for M in LARGE_ROWS:
            s, rows = pick(M, N, K, group), 16 if M <= 16 else 32
            if s.tc:
                units, at_once = -(-N // 128) * -(-M // rows), 148 // s.tc
                seen.add((s.tc, rows, group, "once" if units <= at_once else "in turn"))
            elif s.wn:
                seen.add(("ring", group))
    for group in (32, 64, 128):
        assert ("ring", group) in seen
        for rows in (16, 32):
            assert (1, rows, group, "once") in seen
            for turns in ("once", "in turn"):
                assert (2, rows, group, turns) in seen
        assert (1, 32, group, "in turn") in seen
    assert (1, 16, 32, "in turn") in seen and (1, 16, 64, "in turn") in seen
