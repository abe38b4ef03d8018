"""The scratch that an INT8 weight owns: what a captured graph holds of it, and growth."""

import pytest

from paper_2608_02703_gb300 import archead

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _build():
    from paper_2608_02703_gb300.build import build

    build()


def _weight(N, K):
    import torch

    g = torch.Generator(device="cuda").manual_seed(N)
    codes = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    return archead.archead_int8_weight_create(codes, torch.full((N,), 0.01, device="cuda"))


class _Captured:
    """A product of M activations in a graph, on buffers of its own."""

    def __init__(self, w, M):
        import torch

        self.w, self.M = w, M
        self.x = torch.randn((M, w.K), device="cuda")
        self.y = torch.empty((M, w.N), device="cuda")
        self.run()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.run()

    def run(self):
        archead.archead_int8_linear(self.w, self.x, self.M, self.y)

    def check(self):
        import torch

        self.x.normal_()
        self.y.fill_(float("nan"))
        self.graph.replay()
        torch.cuda.synchronize()
        got = self.y.clone()
        self.run()
        assert torch.equal(got, self.y)
        assert archead.archead_int8_sync_status(self.w) == archead.OK


@pytest.mark.parametrize("sizes", [(8, 512), (8, 70, 2000), (64, 65, 66, 67, 5000), (300, 301)], ids=str)
def test_graphs_replay_after_growth(sizes):
    """Every growth keeps what a graph was given; what is kept is no more than what is in use."""
    import torch

    w = _weight(200, 4096)
    empty = archead.archead_int8_device_bytes(w)
    graphs, held = [], []
    for M in sizes:
        graphs.append(_Captured(w, M))
        held.append(archead.archead_int8_device_bytes(w))
    # The host's account first: nothing is replayed into memory that is not the weight's any more.
    x, y = torch.randn((6000, 4096), device="cuda"), torch.empty((6000, 200), device="cuda")
    archead.archead_int8_linear(w, x, 6000, y)
    now = archead.archead_int8_device_bytes(w)
    need = 6000 * 4096 * 2
    assert now >= held[-1] + need
    assert all(a <= b for a, b in zip(held, held[1:]))
    fill = [torch.full((1 << 22,), 7, dtype=torch.int8, device="cuda") for _ in range(40)]  # (takes what was freed)
    for g in graphs + graphs[::-1]:
        g.check()
    assert archead.archead_int8_device_bytes(w) == now
    assert all(bool((f == 7).all()) for f in fill)
    assert now - empty <= 4 * (need + 6000 * 4 + 512)
    for g in graphs:
        g.graph.reset()
    w.close()


def test_what_no_graph_holds_is_freed():
    import torch

    w = _weight(200, 4096)
    base = archead.archead_int8_device_bytes(w)
    room = 64 * 4096 * 2 + 64 * 4
    x, y = torch.randn((600, 4096), device="cuda"), torch.empty((600, 200), device="cuda")
    archead.archead_int8_linear(w, x, 600, y)
    assert archead.archead_int8_device_bytes(w) == base - room + 600 * 4096 * 2 + (600 * 4 + 255) // 256 * 256
    w.close()


def _too_much(w):
    """A call whose scratch no device has (2^30 tokens of 1024 codes: 2 TB); nothing is queued."""
    import torch

    small = torch.zeros((1, w.K), device="cuda")
    y = torch.zeros((1, w.N), device="cuda")
    return archead.load().archead_int8_linear(w.handle, small.data_ptr(), archead.DTYPE_FP32, 1 << 30, w.K,
                                              y.data_ptr(), archead.DTYPE_FP32, w.N, None)


def test_a_failed_growth_is_the_failed_calls_alone():
    import torch

    w = _weight(256, 1024)
    x, y = torch.randn((40, 1024), device="cuda"), torch.empty((40, 256), device="cuda")
    archead.archead_int8_linear(w, x, 40, y)
    want = y.clone()
    assert _too_much(w) == archead.ERR_OOM
    y.fill_(float("nan"))
    archead.archead_int8_linear(w, x, 40, y)  # (not the failure of the call before)
    assert archead.archead_int8_sync_status(w) == archead.OK and torch.equal(y, want)
    w.close()


def test_room_after_a_failed_growth():
    """What a weight that could not grow has room for is what it says: a call leaves room for smaller ones again."""
    import torch

    w = _weight(256, 1024)
    x, y = torch.randn((40, 1024), device="cuda"), torch.empty((40, 256), device="cuda")
    archead.archead_int8_linear(w, x, 40, y)
    want = y.clone()
    new = archead.archead_int8_device_bytes(w)
    assert _too_much(w) == archead.ERR_OOM
    assert archead.archead_int8_device_bytes(w) < new
    archead.archead_int8_linear(w, x, 20, y)
    assert archead.archead_int8_device_bytes(w) == new  # (room for 64 tokens, as a new weight's)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        archead.archead_int8_linear(w, x, 40, y)
    y.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    graph.reset()
    w.close()


@pytest.mark.parametrize("which", ["stream", "address", "default", "current"])
def test_a_weight_of_strided_codes_filled_in_another_stream(which):
    """Codes and scales that do not lie side by side are copied in the stream that the call was given."""
    import torch

    N, K, M = 96, 160, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    wanted = torch.randint(-128, 128, (K, N), generator=g, device="cuda", dtype=torch.int8)
    codes, scales = torch.zeros((K, N), dtype=torch.int8, device="cuda"), torch.zeros((N, 2), device="cuda")
    x = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    side = torch.cuda.default_stream() if which == "default" else torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
        codes.copy_(wanted)
        scales.fill_(1.0)

    def create():
        stream = dict(stream=side, address=side.cuda_stream, default=side, current=None)[which]
        return archead.archead_int8_weight_create(codes.t(), scales[:, 0], stream=stream)

    if which == "current":
        with torch.cuda.stream(side):
            w = create()
    else:
        with torch.cuda.stream(torch.cuda.Stream()):
            w = create()
    y = torch.empty((M, N), device="cuda")
    archead.archead_int8_matmul(w, x, torch.ones(M, device="cuda"), M, y)
    assert torch.equal(y.double(), x.double() @ wanted.double())
    w.close()
