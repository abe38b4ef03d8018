"""The protocols of the INT8 product's kernels: blocks that share K through one another's shared memory,
and waits that give up."""

import pytest

from paper_2608_02703_gb300 import archead

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _build():
    from paper_2608_02703_gb300.build import build

    build()


def _operands(M, N, K, seed=0):
    """Codes on the device whose sums stay below 2^24, and the sums."""
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    x = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    want = x.double() @ codes.double().t()
    assert float(want.abs().max()) < 2 ** 24
    return codes, x, want


@pytest.mark.parametrize("M", [17, 40, 64, 65, 100, 128])
@pytest.mark.parametrize("N,K", [(100, 1024), (128, 512), (1000, 1000), (2400, 1024), (4000, 512), (300, 1100)], ids=str)
def test_blocks_of_a_stage_or_two_join(M, N, K):
    """K cut into parts of one or two stages: a block sends its sums as soon as it can after its start."""
    import torch

    codes, x, want = _operands(M, N, K, seed=M)
    w = archead.archead_int8_weight_create(codes, torch.ones(N, device="cuda"))
    ones = torch.ones(M, device="cuda")
    ys = [torch.full((M, N), float("nan"), device="cuda") for _ in range(20)]
    for y in ys:  # (back to back)
        archead.archead_int8_matmul_path(w, x, ones, M, y, archead.PATH_PREFILL)
    assert archead.archead_int8_sync_status(w) == archead.OK
    for y in ys:
        assert torch.equal(y.double(), want)
    w.close()


@pytest.fixture(scope="module")
def long_row():
    """Work of some milliseconds in one block: the quantisation of a single long row.  It lets the kernel behind it
    start at once, whose warps that need what it computes then wait for its end, and others for those."""
    import torch

    x = torch.zeros((1, 1 << 28), dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    return lambda: archead.archead_int8_quantize_tokens(x, codes, scales)


@pytest.mark.parametrize("M,N,K", [(1, 40000, 4096), (8, 30000, 2048), (16, 20000, 2501), (3, 20000, 9000)], ids=str)
def test_few_tokens_a_wait_that_gives_up(M, N, K, long_row):
    """The copying warp waits for slots that nobody frees meanwhile (a block has more stages than the twelve slots of
    the largest ring): with a limit of a few cycles it gives up, the call ends, the status says so, and the weight is
    as good as before once the limit is back."""
    import torch

    codes, x, want = _operands(M, N, K, seed=M)
    w = archead.archead_int8_weight_create(codes, torch.ones(N, device="cuda"))
    ones, y = torch.ones(M, device="cuda"), torch.empty((M, N), device="cuda")

    def call():
        y.fill_(float("nan"))
        long_row()
        archead.archead_int8_matmul_path(w, x, ones, M, y, archead.PATH_DECODE)
        return archead.archead_int8_sync_status(w)

    assert call() == archead.OK and torch.equal(y.double(), want)
    for budget in (1, 1000, 100000):
        archead.archead_int8_set_wait_budget(w, budget)
        for _ in range(3):
            assert call() == archead.ERR_DEVICE_TIMEOUT
        archead.archead_int8_set_wait_budget(w, 2_000_000_000)
        assert call() == archead.OK and torch.equal(y.double(), want)
    w.close()


@pytest.mark.parametrize("M,N,K", [(17, 128, 131071), (64, 9728, 131071), (64, 19456, 131071), (128, 1000, 131071),
                                   (128, 19456, 131071), (256, 19456, 131071)], ids=str)
def test_many_tokens_a_wait_that_gives_up(M, N, K):
    """The epilogue waits for a unit's whole K: with a limit of a few cycles it gives up while copies, conversions
    and products are under way.  The call ends without waiting for what nobody completes any more (a limit of a
    second each), the status says so, and the weight is as good as before once the limit is back."""
    import time

    import torch

    g = torch.Generator(device="cuda").manual_seed(M)
    codes = torch.randint(-8, 9, (N, K), generator=g, device="cuda", dtype=torch.int8)
    x = torch.randint(-8, 9, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = archead.archead_int8_weight_create(codes, torch.ones(N, device="cuda"))
    rows = torch.arange(0, N, max(1, N // 500), device="cuda")
    want = x.double() @ codes[rows].double().t()  # (exact below 2^24)
    assert float(want.abs().max()) < 2 ** 24
    del codes
    ones, y = torch.ones(M, device="cuda"), torch.empty((M, N), device="cuda")

    def call():
        y.fill_(float("nan"))
        torch.cuda.synchronize()
        t = time.perf_counter()
        archead.archead_int8_matmul_path(w, x, ones, M, y, archead.PATH_PREFILL)
        status = archead.archead_int8_sync_status(w)
        return status, time.perf_counter() - t

    def is_right():
        return call()[0] == archead.OK and torch.equal(y[:, rows].double(), want)

    assert is_right()
    for budget in (1, 1000):
        archead.archead_int8_set_wait_budget(w, budget)
        for _ in range(3):
            status, seconds = call()
            assert status == archead.ERR_DEVICE_TIMEOUT and seconds < 0.3
        archead.archead_int8_set_wait_budget(w, 2_000_000_000)
        assert is_right()
    w.close()
