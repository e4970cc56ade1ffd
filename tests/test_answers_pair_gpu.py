"""Layers on codes by pairs of CTAs: launches directly behind one another, hand-overs over many short tiles (needs a
GPU)."""
import pytest

pytestmark = pytest.mark.gpu


def layer(gpu_lib, rows, n_in, n_out, seed):
    """Codes with scales of one, whose sums are exact in fp32 (below 2^24), and those sums."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-127, 128, (rows, n_in), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (n_out, n_in), generator=g, device="cuda").to(torch.int8)
    xs, ws = torch.ones(rows, device="cuda"), torch.ones(n_out, device="cuda")
    want = (x.double() @ w.double().T).float()
    # rows on 16-byte boundaries: of the kernels, only the pairs' takes workspace
    n = gpu_lib.mca_code_linear_workspace_size(x, xs, w, ws)
    assert n > 0
    return (x, xs, w, ws), want, torch.empty(n, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("rows,n_in,n_out", [(2048, 64, 8192), (3001, 48, 9001), (1500, 1024, 3000),
                                             (900, 1040, 5000)])
def test_pairs_behind_one_another(gpu_lib, rows, n_in, n_out):
    """One to seventeen chunks of columns a tile, two to some dozens of tiles a pair: each launch follows the last
    on SMs that it has just left, with another kernel's shared memory in between."""
    import torch
    a, want_a, ws_a = layer(gpu_lib, rows, n_in, n_out, 1)
    b, want_b, ws_b = layer(gpu_lib, rows // 2 * 2, n_in, n_out, 2)
    few = (a[0][:48].contiguous(), a[1][:48], a[2], a[3])
    ya = [torch.full_like(want_a, float("nan")) for _ in range(6)]
    yb = [torch.full_like(want_b, float("nan")) for _ in range(6)]
    yf = [torch.full_like(want_a[:48], float("nan")) for _ in range(6)]
    for i in range(6):
        gpu_lib.mca_code_linear(*a, out=ya[i], workspace=ws_a)
        gpu_lib.mca_code_linear(*few, out=yf[i])
        gpu_lib.mca_code_linear(*b, out=yb[i], workspace=ws_b)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want_a) for y in ya)
    assert all(torch.equal(y, want_a[:48]) for y in yf)
    assert all(torch.equal(y, want_b) for y in yb)


def test_pairs_on_two_streams(gpu_lib):
    """Two layers at once, each with its own workspace."""
    import torch
    made = [layer(gpu_lib, 2048, 64, 8192, 3), layer(gpu_lib, 1200, 2000, 3001, 4)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    out = [[torch.full_like(want, float("nan")) for _ in range(8)] for _, want, _ in made]
    torch.cuda.synchronize()
    for i in range(8):
        for (arg, _, ws), ys, st in zip(made, out, streams):
            gpu_lib.mca_code_linear(*arg, out=ys[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    for (_, want, _), ys in zip(made, out):
        assert all(torch.equal(y, want) for y in ys)


def test_all_kernels_at_once(gpu_lib):
    """The three kernels on three streams, on each other's SMs: few samples, some dozens with the columns over clusters,
    many."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    made = [layer(gpu_lib, 2048, 64, 8192, 5)]
    for rows, n_in, n_out in ((4, 4096, 16384), (48, 16000, 700), (64, 4096, 2048), (120, 8192, 1000)):
        x = torch.randint(-127, 128, (rows, n_in), generator=g, device="cuda").to(torch.int8)
        w = torch.randint(-127, 128, (n_out, n_in), generator=g, device="cuda").to(torch.int8)
        one = torch.ones(max(rows, n_out), device="cuda")
        arg = (x, one[:rows], w, one[:n_out])
        assert gpu_lib.mca_code_linear_workspace_size(*arg) == 0
        made.append((arg, (x.double() @ w.double().T).float(), None))
    streams = [torch.cuda.Stream() for _ in made]
    out = [[torch.full_like(want, float("nan")) for _ in range(12)] for _, want, _ in made]
    torch.cuda.synchronize()
    for i in range(12):
        for (arg, _, ws), ys, st in zip(made, out, streams):
            gpu_lib.mca_code_linear(*arg, out=ys[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    for (_, want, _), ys in zip(made, out):
        assert all(torch.equal(y, want) for y in ys)


def test_two_graphs_of_pairs(gpu_lib):
    """Two captured layers replayed at the same time: each has the images of its own operands."""
    import torch
    made = []
    for seed, rows, n_in, n_out in ((8, 2048, 64, 8192), (9, 1200, 2000, 3001)):
        arg, want, _ = layer(gpu_lib, rows, n_in, n_out, seed)
        gpu_lib.mca_code_linear(*arg)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = gpu_lib.mca_code_linear(*arg)
        made.append((graph, y, want, torch.cuda.Stream(), arg))
    torch.cuda.synchronize()
    for _ in range(10):
        for graph, y, _, st, _ in made:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, y, want, *_ in made:
        assert torch.equal(y, want)
