"""The answers' operators on a stream that is not the current one: the tensors given are kept until their work is done."""
import contextlib
from types import SimpleNamespace

import pytest

from paper_2607_08406_gb300 import mca


class Given:
    def __init__(self):
        self.on = []

    def record_stream(self, st):
        self.on.append(st)


def fake_torch(current):
    @contextlib.contextmanager
    def entered(*_):
        yield
    cuda = SimpleNamespace(device=entered, stream=entered, ExternalStream=lambda s: ("stream", s),
                           default_stream=lambda: ("stream", 0),
                           current_stream=lambda: SimpleNamespace(cuda_stream=current))
    return SimpleNamespace(cuda=cuda, _C=SimpleNamespace(_cuda_getDevice=lambda: 0,
                                                         _cuda_getCurrentRawStream=lambda i: current))


@pytest.mark.parametrize("index", [0, 1])
@pytest.mark.parametrize("stream,kept", [(None, []), (5, []), (7, [("stream", 7)]), (0, [("stream", 0)]),
                                         (SimpleNamespace(cuda_stream=7), [("stream", 7)])])
def test_given_tensors_are_recorded(monkeypatch, stream, kept, index):
    monkeypatch.setattr(mca, "torch", fake_torch(current=5))
    given = [Given(), None, Given()]
    assert mca._on(index, stream, given, lambda s: s) == (5 if not kept else kept[0][1])
    assert given[0].on == kept and given[2].on == kept

    def failing(s):
        raise RuntimeError("after a first launch")
    with pytest.raises(RuntimeError):
        mca._on(index, stream, given, failing)
    assert given[0].on == 2 * kept


def calls(lib):
    """Each operator with every tensor it may be given: (name, inputs, call(inputs, stream))."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    rows, n_in, n_out, V = 64, 256, 512, 3000
    x = torch.randn(rows, n_in, generator=g, device="cuda")
    q, s = lib.mca_quantize_rows(x)
    w = torch.randint(-127, 128, (n_out, n_in), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand(n_out, generator=g, device="cuda")
    b = torch.rand(n_out, generator=g, device="cuda")
    z = torch.randn(rows, V, generator=g, device="cuda")
    t = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    r = lib.mca_token_logprobs(z, t)
    gl, ge = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    return [("quantize", [x], lambda a, st: lib.mca_quantize_rows(*a, stream=st)),
            ("linear", [q, s, w, ws, b], lambda a, st: [lib.mca_code_linear(*a, stream=st)]),
            ("score", [z, t], lambda a, st: list(lib.mca_token_logprobs(*a, top=3, stream=st))),
            ("grad", [z, t, r.lse, r.entropy, gl, ge],
             lambda a, st: [lib.mca_token_logprobs_backward(*a, stream=st)])]


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("raw", [False, True])
def test_inputs_freed_while_their_work_waits(gpu_lib, which, raw):
    """Inputs that the caller lets go of while the work waits on a busy stream: their memory is not handed out, and
    the results are those of the inputs."""
    import torch
    name, args, call = calls(gpu_lib)[which]
    want = call(args, None)
    side = torch.cuda.Stream()
    busy = torch.randn(8192, 8192, device="cuda").to(torch.bfloat16)
    other = torch.empty_like(busy)
    mine = [a.clone() for a in args]
    sizes = [(a.shape, a.dtype, a.data_ptr()) for a in mine]
    # kernels and memory for what comes, whose first use could wait for the device
    call(args, side)
    for st in (side, torch.cuda.current_stream()):
        with torch.cuda.stream(st):
            spare = [torch.full((1 << 19,), 1, dtype=dt, device="cuda")
                     for dt in (torch.int8, torch.int32, torch.float32) for _ in range(8)]
            torch.matmul(busy, busy, out=other)
            del spare
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(60):                                  # some 40 ms
            torch.matmul(busy, busy, out=other)
    got = call(mine, side.cuda_stream if raw else side)
    del mine
    again = [torch.full(shape, 1, dtype=dt, device="cuda") for shape, dt, _ in sizes]
    assert not side.query(), "the work was not waiting any more"
    assert not {a.data_ptr() for a in again} & {p for _, _, p in sizes}, name
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want)), name


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [33, 2048])
def test_captured_on_another_stream(gpu_lib, rows):
    """The chain on a stream that a capture has taken in, replayed on new inputs: bit for bit the eager results."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    n_in, vocab = 256, 3001
    xs = [torch.randn(rows, n_in, generator=g, device="cuda") for _ in range(2)]
    w = torch.randint(-127, 128, (vocab, n_in), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand(vocab, generator=g, device="cuda") * 1e-3
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)

    def chain(x, stream):
        q, s = gpu_lib.mca_quantize_rows(x, stream=stream)
        y = gpu_lib.mca_code_linear(q, s, w, ws, dtype=torch.float16, stream=stream)
        r = gpu_lib.mca_token_logprobs(y, t, top=4, stream=stream)
        return [q, s, y, *r, gpu_lib.mca_token_logprobs_backward(y, t, r.lse, r.entropy, r.logprob, r.entropy,
                                                                 stream=stream)]
    want = [chain(x, None) for x in xs]
    buf, side, graph = xs[0].clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = chain(buf, side)
        torch.cuda.current_stream().wait_stream(side)
    for x, ref in ((xs[1], want[1]), (xs[0], want[0])):
        buf.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
