"""The INT8 product and its quantiser against their definitions in 64 bits.

Bounds.  The quantiser is defined in fp32 operations, which numpy does the
same: codes and scales are equal.  A product's sum of integers is exact (or,
beyond 2^24, within the fp32 roundings counted below); turning it into fp32
and two products with scales are three roundings of 2^-24 of the value each,
the output's rounding is 2^-8 (bf16), 2^-11 (fp16, 2^-25 absolute below its
normal range) or none (fp32).
"""

import numpy as np
import pytest

from paper_2608_02703_gb300 import archead

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 0.0}


@pytest.fixture(scope="module", autouse=True)
def _build():
    from paper_2608_02703_gb300.build import build

    build()


def _torch():
    import torch

    return torch


def _dtype(name):
    torch = _torch()
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def _quantized(x):
    """The definition, in numpy's fp32."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x), np.float32)
        s = amax / np.float32(127)
        usable = np.isfinite(s) & (s > 0)
        q = np.clip(np.rint(x / np.where(usable, s, np.float32(1))[:, None]), -127, 127)
    return np.where(usable[:, None], q, 0).astype(np.int8), s


def _draw(M, N, K, seed):
    rng = np.random.default_rng(seed)
    codes = rng.integers(-128, 128, (N, K), dtype=np.int8)
    scales = (rng.uniform(0.5, 2, N) * 0.01).astype(np.float32)
    x_codes = rng.integers(-128, 128, (M, K), dtype=np.int8)
    x_scales = (rng.uniform(0.5, 2, M) * 0.02).astype(np.float32)
    return codes, scales, x_codes, x_scales


def _want(codes, scales, x_codes, x_scales):
    sums = x_codes.astype(np.float64) @ codes.astype(np.float64).T
    return sums * x_scales.astype(np.float64)[:, None] * scales.astype(np.float64)[None, :]


def _check(y, want, out, more=0.0):
    got = y.double().cpu().numpy()
    bound = (DTYPES[out] + 3.1 * 2.0 ** -24 + more) * np.abs(want) + (2.0 ** -25 if out == "fp16" else 2.0 ** -140)
    off = np.abs(got - want) - bound
    assert off.max() <= 0, f"worst at {np.unravel_index(off.argmax(), off.shape)}: {off.max():.3e} over its bound"


def _dev(a):
    return _torch().from_numpy(np.ascontiguousarray(a)).cuda()


# ------------------------------------------------------------------------
# Quantiser
# ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("M,K,ldx", [(1, 1, 1), (1, 17, 17), (3, 31, 40), (5, 512, 512), (2, 4096, 4096), (7, 2501, 2503),
                                     (300, 640, 640), (2, 40000, 40000), (65, 8192, 8200)])
def test_quantize_equals_definition(dtype, M, K, ldx):
    torch = _torch()
    g = torch.Generator().manual_seed(M * 1000 + K)
    x = (torch.randn((M, ldx), generator=g) * torch.exp2(torch.rand(M, 1, generator=g) * 20 - 12)).to(_dtype(dtype))
    x = x[:, :K]
    codes = torch.full((M, K), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((M,), -1.0, device="cuda")
    whole = x.cuda() if ldx == K else torch.nn.functional.pad(x, (0, ldx - K), value=1e4).cuda()[:, :K]
    archead.archead_int8_quantize_tokens(whole, codes, scales)
    want, s = _quantized(x.float().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("K", [1, 7, 8, 9, 241, 248, 249, 985, 992, 993, 1985, 3968, 7929, 7936, 7951, 9001])
def test_quantize_rows_on_any_element(dtype, K):
    """Rows that start on every element of 16 bytes and end on every one: what lies
    between rows does not count, what lies around the codes is not written."""
    torch = _torch()
    g = torch.Generator().manual_seed(K)
    for offset in range(4 if dtype == "fp32" else 8):
        M, ldx = 9, K + (0, 1, 3, 4)[(offset + K) % 4]
        x = torch.randn((M, K), generator=g).to(_dtype(dtype))
        buf = torch.full((offset + M * ldx + 16,), float("nan") if offset % 2 else 3e4, dtype=_dtype(dtype))
        rows = buf[offset:offset + M * ldx].view(M, ldx)
        rows[:, :K] = x
        on_gpu = buf.cuda()
        out = torch.full((16 + M * K + 16,), 99, dtype=torch.int8, device="cuda")
        codes, scales = out[16:16 + M * K].view(M, K), torch.full((M,), -1.0, device="cuda")
        archead.archead_int8_quantize_tokens(on_gpu[offset:offset + M * ldx].view(M, ldx)[:, :K], codes, scales)
        want, s = _quantized(x.float().numpy())
        np.testing.assert_array_equal(scales.cpu().numpy(), s)
        np.testing.assert_array_equal(codes.cpu().numpy(), want)
        assert bool((out[:16] == 99).all()) and bool((out[16 + M * K:] == 99).all())


def test_quantize_edge_rows():
    """Zero rows, values at half steps (ties to even), the smallest and largest scales, infinities and NaNs."""
    torch = _torch()
    K = 264
    rows = np.zeros((12, K), np.float32)
    rows[1] = -0.0
    rows[2, :255] = (np.arange(255) - 127) / 2  # steps of half a code (scale 0.5)
    rows[3] = rows[2] * np.float32(2.0 ** -126)
    rows[4, 5] = 1e-44  # scale rounds to zero
    rows[5] = 1e-45 * 190  # scale of one step of the subnormals: codes are clamped
    rows[6] = np.linspace(-3.4e38, 3.4e38, K)
    rows[7, 3], rows[7, 9] = np.inf, 2
    rows[8, K - 1] = np.nan
    rows[9, 0] = -np.inf
    rows[10] = np.linspace(-1, 1, K)
    rows[11] = np.where(np.arange(K) % 2, 1.5, -63.5) * np.float32(2 ** -140)
    codes = torch.empty((12, K), dtype=torch.int8, device="cuda")
    scales = torch.empty(12, device="cuda")
    archead.archead_int8_quantize_tokens(_dev(rows), codes, scales)
    want, s = _quantized(rows)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy(), want)
    assert np.isinf(s[7]) and np.isnan(s[8]) and not want[7:10].any() and not want[4].any()


def test_quantize_every_bf16_value():
    torch = _torch()
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    x = np.stack([x[np.isfinite(x) & (np.abs(x) <= 2.0 ** e)][:16000] for e in (0, 10, -20)])
    t = torch.from_numpy(x).cuda().to(torch.bfloat16)
    codes = torch.empty(t.shape, dtype=torch.int8, device="cuda")
    scales = torch.empty(3, device="cuda")
    archead.archead_int8_quantize_tokens(t, codes, scales)
    want, s = _quantized(x)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)
    np.testing.assert_array_equal(codes.cpu().numpy(), want)


# ------------------------------------------------------------------------
# Product
# ------------------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 16, 32), (1, 4096, 512), (2, 130, 33), (8, 128, 128), (9, 257, 640), (5, 17, 4096),
         (16, 1000, 2501), (17, 384, 256), (31, 129, 1), (32, 300, 31), (33, 512, 320), (64, 1024, 576),
         (65, 130, 1000), (100, 1003, 2501), (128, 256, 128), (129, 640, 384), (200, 127, 130), (256, 2000, 512),
         (257, 129, 96), (300, 256, 8192), (511, 300, 300), (700, 70, 200), (1025, 260, 257)]
PATHS = {"auto": archead.PATH_AUTO, "decode": archead.PATH_DECODE, "prefill": archead.PATH_PREFILL}


@pytest.mark.parametrize("path", list(PATHS))
@pytest.mark.parametrize("M,N,K", SIZES, ids=str)
def test_product(M, N, K, path):
    torch = _torch()
    a = _draw(M, N, K, seed=M + N + K)
    w = archead.archead_int8_weight_create(a[0], a[1])
    out = ("bf16", "fp16", "fp32")[(M + N + K) % 3]
    for dt in {out, "fp32"}:
        y = torch.full((M, N), float("nan"), dtype=_dtype(dt), device="cuda")
        archead.archead_int8_matmul_path(w, _dev(a[2]), _dev(a[3]), M, y, PATHS[path])
        assert archead.archead_int8_sync_status(w) == archead.OK
        _check(y, _want(*a), dt)
    w.close()


@pytest.mark.parametrize("path", list(PATHS))
@pytest.mark.parametrize("M", [1, 7, 16, 24, 40, 64, 100, 129, 300])
@pytest.mark.parametrize("N,K", [(4096, 512), (1500, 4096), (20000, 256)], ids=str)
def test_product_split_and_whole(M, N, K, path):
    """Widths at which K is split over blocks, and at which it is not."""
    torch = _torch()
    a = _draw(M, N, K, seed=M + K)
    w = archead.archead_int8_weight_create(a[0], a[1])
    y = torch.full((M, N), float("nan"), dtype=torch.float32, device="cuda")
    for _ in range(3):  # (counters and scratch are as a call before left them)
        y.fill_(float("nan"))
        archead.archead_int8_matmul_path(w, _dev(a[2]), _dev(a[3]), M, y, PATHS[path])
        _check(y, _want(*a), "fp32")
    assert archead.archead_int8_sync_status(w) == archead.OK
    w.close()


@pytest.mark.parametrize("M", [1, 3, 8, 9, 16])
@pytest.mark.parametrize("N,K", [(9760, 2001), (10007, 1303), (19473, 200), (20000, 1024), (39000, 640)], ids=str)
def test_few_tokens_in_rounds_of_two_kinds(M, N, K):
    """Channels that all multiprocessors take in whole rounds, and a rest that is cut along K."""
    torch = _torch()
    a = _draw(M, N, K, seed=N + M)
    w = archead.archead_int8_weight_create(a[0], a[1])
    y = torch.full((M, N), float("nan"), dtype=torch.float32, device="cuda")
    archead.archead_int8_matmul_path(w, _dev(a[2]), _dev(a[3]), M, y, archead.PATH_DECODE)
    _check(y, _want(*a), "fp32")
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).to(torch.bfloat16)
    q, s = _quantized(x.float().numpy())
    archead.archead_int8_linear(w, x.cuda(), M, y)
    _check(y, _want(a[0], a[1], q, s), "fp32")
    assert archead.archead_int8_sync_status(w) == archead.OK
    w.close()


@pytest.mark.parametrize("M", [1, 8, 20, 40, 64, 100, 128, 200, 300])
def test_wide_weights_from_memory(M):
    """Many units a block, whose codes come from memory (more of them than the second-level cache holds) and so in any
    order; repeated."""
    torch = _torch()
    N, K = 70000, 2304
    g = torch.Generator(device="cuda").manual_seed(M)
    codes = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    x = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = archead.archead_int8_weight_create(codes, torch.ones(N, device="cuda"))
    # Sums below 2^24 are exact: 64-bit products of the codes, rows at a time.
    want = torch.cat([x.double() @ codes[n:n + 10000].double().t() for n in range(0, N, 10000)], dim=1)
    assert float(want.abs().max()) < 2 ** 24
    y = torch.empty((M, N), device="cuda")
    for _ in range(6):
        y.fill_(float("nan"))
        archead.archead_int8_matmul(w, x, torch.ones(M, device="cuda"), M, y)
        assert archead.archead_int8_sync_status(w) == archead.OK
        assert torch.equal(y.double(), want)
    w.close()


@pytest.mark.parametrize("path", list(PATHS))
@pytest.mark.parametrize("M,K", [(3, 131071), (20, 40000), (70, 20000), (140, 5000)], ids=str)
def test_largest_sums(M, K, path):
    """All codes of one sign and the largest size.  The warp-level kernel's
    sums are exact integers up to 8 tokens; otherwise sums beyond 2^24 are
    rounded to fp32: an addition of 16 products (at most K / 16 in turn, on
    sums that grow evenly: half the last one's size on average) loses at most
    one unit in the last place, 2^-23 of the sum."""
    torch = _torch()
    N = 40
    codes = np.full((N, K), -128, np.int8)
    codes[1::2] = 127
    x = np.full((M, K), 127, np.int8)
    x[1::3] = -128
    scales, x_scales = np.full(N, 2.0 ** -10, np.float32), np.full(M, 2.0 ** -9, np.float32)
    w = archead.archead_int8_weight_create(codes, scales)
    y = torch.empty((M, N), device="cuda")
    archead.archead_int8_matmul_path(w, _dev(x), _dev(x_scales), M, y, PATHS[path])
    assert archead.archead_int8_sync_status(w) == archead.OK
    want = _want(codes, scales, x, x_scales)
    exact = M <= 8 and path != "prefill"
    _check(y, want, "fp32", more=0.0 if exact else K / 16 * 2.0 ** -24)
    w.close()


@pytest.mark.parametrize("path", list(PATHS))
def test_single_places(path):
    """One nonzero code on each side: the layouts agree at every place."""
    torch = _torch()
    K, N, M = 200, 150, 70
    rng = np.random.default_rng(3)
    codes = np.zeros((N, K), np.int8)
    codes[np.arange(N), rng.integers(0, K, N)] = rng.integers(1, 128, N)
    x = np.zeros((M, K), np.int8)
    x[:] = (np.arange(K) % 127 + 1)[None, :]
    x[::2] *= -1
    one = (np.ones(N, np.float32), np.ones(M, np.float32))
    w = archead.archead_int8_weight_create(codes, one[0])
    y = torch.empty((M, N), device="cuda")
    archead.archead_int8_matmul_path(w, _dev(x), _dev(one[1]), M, y, PATHS[path])
    np.testing.assert_array_equal(y.cpu().numpy(), _want(codes, one[0], x, one[1]).astype(np.float32))
    w.close()


@pytest.mark.parametrize("x_dtype", list(DTYPES))
@pytest.mark.parametrize("out", list(DTYPES))
@pytest.mark.parametrize("M,N,K", [(1, 300, 100), (8, 2000, 4096), (30, 129, 1111), (90, 1000, 2048), (400, 300, 640)],
                         ids=str)
def test_linear_is_quantisation_then_product(x_dtype, out, M, N, K):
    torch = _torch()
    codes, scales, _, _ = _draw(1, N, K, seed=N)
    g = torch.Generator().manual_seed(M)
    x = torch.randn((M, K), generator=g).to(_dtype(x_dtype))
    x[M // 2] = 0
    w = archead.archead_int8_weight_create(codes, scales)
    y = torch.full((M, N), float("nan"), dtype=_dtype(out), device="cuda")
    archead.archead_int8_linear(w, x.cuda(), M, y)
    q, s = _quantized(x.float().numpy())
    _check(y, _want(codes, scales, q, s), out)
    two = torch.empty_like(y)
    c, sc = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    archead.archead_int8_quantize_tokens(x.cuda(), c, sc)
    archead.archead_int8_matmul(w, c, sc, M, two)
    assert torch.equal(y, two)
    w.close()


@pytest.mark.parametrize("M", [3, 40, 200])
def test_rows_apart(M):
    """Inputs and outputs whose rows are some distance apart; what lies between output rows is not touched."""
    torch = _torch()
    N, K = 131, 203
    codes, scales, _, _ = _draw(1, N, K, seed=5)
    w = archead.archead_int8_weight_create(codes, scales)
    x = torch.randn((M, K + 5), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    for pad in (1, 8, 13):
        whole = torch.full((M, N + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        archead.archead_int8_linear(w, x[:, :K], M, whole[:, :N])
        q, s = _quantized(x[:, :K].float().cpu().numpy())
        _check(whole[:, :N], _want(codes, scales, q, s), "bf16")
        assert bool((whole[:, N:] == 7).all())
    w.close()


@pytest.mark.parametrize("M", [5, 30, 200])
def test_rows_that_are_not_finite(M):
    """A NaN or an infinity in a token makes its outputs NaN and no other's."""
    torch = _torch()
    N, K = 260, 300
    codes, scales, _, _ = _draw(1, N, K, seed=6)
    w = archead.archead_int8_weight_create(codes, scales)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(1)).cuda()
    x[1, 7], x[3, 299] = float("nan"), float("inf")
    y = torch.empty((M, N), device="cuda")
    archead.archead_int8_linear(w, x, M, y)
    bad = torch.isnan(y).any(dim=1).cpu().numpy()
    assert bad[1] and bad[3] and bad.sum() == 2 and bool(torch.isnan(y[[1, 3]]).all())
    w.close()


@pytest.mark.parametrize("M,N,K", [(4, 4096, 1024), (24, 4096, 1024), (96, 4096, 1024), (300, 1000, 1024)], ids=str)
def test_repeats_bit_for_bit_and_on_other_streams(M, N, K):
    torch = _torch()
    a = _draw(M, N, K, seed=8)
    w = archead.archead_int8_weight_create(_dev(a[0]), _dev(a[1]))  # (device arrays)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    ys = [torch.empty((M, N), device="cuda") for _ in range(6)]
    side = torch.cuda.Stream()
    for i, y in enumerate(ys):
        torch.cuda.synchronize()
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            archead.archead_int8_linear(w, x, M, y)
        torch.cuda.synchronize()
    assert archead.archead_int8_sync_status(w) == archead.OK
    for y in ys[1:]:
        assert torch.equal(y, ys[0])
    w.close()


@pytest.mark.parametrize("warm,M", [(1, 1), (1, 64), (300, 300), (300, 70), (300, 9), (1000, 130)])
def test_captured_after_a_warm_up(warm, M):
    """A new weight has room for 64 tokens, a call leaves room for fewer."""
    torch = _torch()
    N, K = 3000, 512
    codes, scales, _, _ = _draw(1, N, K, seed=9)
    w = archead.archead_int8_weight_create(codes, scales)
    g = torch.Generator().manual_seed(2)
    x = torch.randn((max(warm, M), K), generator=g).cuda()
    y = torch.empty((max(warm, M), N), device="cuda")
    other = archead.archead_int8_weight_create(codes, scales)
    want = torch.empty((M, N), device="cuda")
    x2 = torch.randn((M, K), generator=g).cuda()
    archead.archead_int8_linear(other, x2, M, want)  # (loads the kernels)
    archead.archead_int8_linear(w, x, warm, y)
    held = archead.archead_int8_device_bytes(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        archead.archead_int8_linear(w, x, M, y)
    assert archead.archead_int8_device_bytes(w) == held
    x[:M].copy_(x2)
    y.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y[:M], want)
    w.close()
    other.close()


def test_growth_in_a_capture_is_refused():
    torch = _torch()
    codes, scales, _, _ = _draw(1, 200, 4096, seed=9)
    w = archead.archead_int8_weight_create(codes, scales)
    x, y = torch.randn((5000, 4096)).cuda(), torch.empty((5000, 200), device="cuda")
    archead.archead_int8_linear(w, x, 5, y)
    want = y[:5].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
        y.add_(0)
        with pytest.raises(archead.ArcheadError) as e:
            archead.archead_int8_linear(w, x, 5000, y)
        assert e.value.status == archead.ERR_UNSUPPORTED
    archead.archead_int8_linear(w, x, 5, y)
    torch.cuda.synchronize()
    assert torch.equal(y[:5], want)
    w.close()


def test_refusals():
    torch = _torch()
    codes, scales, _, _ = _draw(1, 40, 64, seed=9)
    w = archead.archead_int8_weight_create(codes, scales)
    x, y = torch.zeros((3, 64), device="cuda"), torch.zeros((3, 40), device="cuda")
    lib = archead.load()
    p = lambda t, o=0: t.data_ptr() + o  # noqa: E731
    ok = dict(h=w.handle, x=p(x), xd=1, M=3, ldx=64, y=p(y), od=1, ldy=40)
    for kw, want in ((dict(), archead.OK), (dict(x=None), 1), (dict(y=None), 1), (dict(x=p(x, 4)), 1),
                     (dict(y=p(y, 8)), 1), (dict(M=-1), 1), (dict(ldx=63), 1), (dict(ldy=39), 1), (dict(xd=5), 1),
                     (dict(od=5), 1), (dict(M=0, x=None, y=None), 0), (dict(M=(1 << 30) + 1), archead.ERR_UNSUPPORTED)):
        a = ok | kw
        assert lib.archead_int8_linear(a["h"], a["x"], a["xd"], a["M"], a["ldx"], a["y"], a["od"], a["ldy"], None) == want
    c, s = torch.zeros((3, 64), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    assert lib.archead_int8_matmul_path(w.handle, p(c), p(s), 3, p(y), 1, 40, 3, None) == archead.ERR_INVALID_ARG
    assert lib.archead_int8_matmul(w.handle, p(c), p(s, 4), 3, p(y), 1, 40, None) == archead.ERR_INVALID_ARG
    assert lib.archead_int8_matmul(w.handle, p(c), None, 3, p(y), 1, 40, None) == archead.ERR_INVALID_ARG
    assert lib.archead_int8_set_wait_budget(w.handle, 0) == archead.ERR_INVALID_ARG
    assert archead.archead_int8_sync_status(w) == archead.OK
    w.close()
