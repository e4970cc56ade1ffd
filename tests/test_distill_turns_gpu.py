"""The loss against a teacher's list of many rows that are long, or of the lengths at which another kernel takes over
(needs a GPU); test_row_shapes.py says which kernel has which of these sizes."""
import os
import subprocess
import sys

import numpy as np
import pytest

import drafts_reference as R
from test_answers_gpu import DT, f64, torch_dtype
from test_distill_gpu import close

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def case(seed, rows, vocab, dtype, top, pad=0, offset=0, tail=True):
    """Logits and a teacher's lists on the GPU: half of the listed symbols among the net's largest, lists of all lengths."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch_dtype(dtype)
    buf = torch.full((offset + rows * (vocab + pad) + 32,), float("nan"), dtype=dt, device="cuda")
    x = buf.as_strided((rows, vocab), (vocab + pad, 1), offset)
    x.copy_(2.0 * torch.randn(rows, vocab, generator=g, device="cuda"))
    index = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:top] for _ in range(8)])
    index = index[torch.randint(0, 8, (rows,), generator=g, device="cuda")]
    index = ((index + torch.arange(rows, device="cuda")[:, None] * 37) % vocab).to(torch.int32).contiguous()
    t = torch.log_softmax(2.0 * torch.randn(rows, top + 1, generator=g, device="cuda"), 1)[:, :top].contiguous()
    x.scatter_add_(1, index[:, ::2].long(), t[:, ::2].exp().to(dt) * 4)
    n = torch.randint(0, top + 1, (rows, 1), generator=g, device="cuda")
    n[::3] = top
    none = torch.arange(top, device="cuda") >= n
    index[none] = -1
    t[none] = float("-inf")
    return x, index, t


def check_picked(lib, x, index, teacher, T, tail, pick, dtype, r=None):
    """Loss, and the gradient, of rows `pick` against the reference."""
    import torch
    r = lib.mca_distill(x, index, teacher, T, tail=tail) if r is None else r
    xs, ii, tt = f64(x[pick]), index[pick].cpu().numpy(), f64(teacher[pick])
    w = R.distill(xs, ii, tt, T, tail)
    for name in ("lse", "loss") + (("rest",) if tail else ()):
        close(getattr(r, name)[pick], w[name], w["tol_" + name])
    d = lib.mca_distill_backward(x, index, teacher, r.lse, torch.ones_like(r.lse), T, rest=r.rest)
    gw, gt = R.distill_backward(xs, ii, tt, T, tail, f64(r.lse[pick]), f64(r.rest[pick]) if tail else None,
                                np.ones(len(xs)), dtype)
    if dtype == "float16":                                       # (beyond its range)
        gw = np.where(np.abs(gw) >= 65520.0, np.copysign(np.inf, gw), gw)
    close(d[pick], gw, gt)
    return r


# ------------------------------------------------------------------------------------------------
# rows in shared memory, up to their largest
# ------------------------------------------------------------------------------------------------

# pieces of 16 bytes of the longest row: around 2048, 48 kB of them, and the most that a row in shared memory may have
LEAST, OPT_IN, MOST = 2048, (48 << 10) // 16, 3200
PIECES = [("least", -1), ("least", 0), ("least", 1), ("opt_in", -2), ("opt_in", -1), ("opt_in", 0), ("opt_in", 1),
          ("most", -1), ("most", 0), ("most", 1)]


def pieces_of(border, more):
    return {"least": LEAST, "opt_in": OPT_IN, "most": MOST}[border] + more


def vocab_of(pieces, dtype, last=False):
    """The shortest, or longest, vocabulary whose rows have so many pieces wherever they start."""
    n = 4 if dtype == "float32" else 8
    return n * pieces - 2 * n + 2 + (n - 1 if last else 0)


@pytest.mark.parametrize("more", [-1, 0])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_first_call_of_a_process(gpu_lib, dtype, more):
    """Rows whose shared memory is just above what a launch has without asking for more, in a process that has had no
    longer ones."""
    code = ("import torch\nfrom paper_2607_08406_gb300 import mca\n"
            f"x = torch.zeros(620, {vocab_of(OPT_IN + more, dtype, True)}, dtype=torch.{dtype}, device='cuda')\n"
            "i = torch.zeros(620, 1, dtype=torch.int32, device='cuda')\n"
            "r = mca.mca_distill(x, i, torch.full((620, 1), -0.5, device='cuda'), tail=True)\n"
            "assert bool(torch.isfinite(r.loss).all())\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("border,more", PIECES)
@pytest.mark.parametrize("last", [False, True])
def test_pieces_at_the_borders(gpu_lib, dtype, border, more, last):
    import torch
    pieces = pieces_of(border, more)
    rows, vocab = 611, vocab_of(pieces, dtype, last)
    for tail, pad in ((True, 0), (True, 3), (False, 1)):
        x, index, t = case(pieces + pad, rows, vocab, dtype, 24, pad, pad)
        index[7] = index[7, 0]                                   # one symbol throughout
        x[8] = float("-inf")
        x[9, vocab - 1] = float("nan")
        x[10, : vocab - 2] = float("-inf")
        check_picked(gpu_lib, x, index, t, 1.0, tail, torch.tensor([0, 1, 7, 8, 9, 10, 304, rows - 1], device="cuda"), dtype)


IN_BETWEEN = [(1300, 16380, "bfloat16"), (1300, 16383, "float16"), (1300, 8190, "float32"), (2500, 16378, "bfloat16"),
              (2500, 8191, "float32")]


@pytest.mark.parametrize("rows,vocab,dtype", IN_BETWEEN)
def test_rows_too_long_for_shared_memory_and_too_short_to_stay(gpu_lib, rows, vocab, dtype):
    import torch
    x, index, t = case(vocab, rows, vocab, dtype, 24, 1, 1)
    x[8] = float("-inf")
    x[9, vocab - 1] = float("nan")
    x[10, : vocab - 2] = float("-inf")
    check_picked(gpu_lib, x, index, t, 1.0, False, torch.tensor([0, 1, 8, 9, 10, 1299, rows - 1], device="cuda"), dtype)


# ------------------------------------------------------------------------------------------------
# CTAs that stay: two and three rows to each, some with one less
# ------------------------------------------------------------------------------------------------

STAYING = [(912, 16390, "bfloat16", False), (1300, 16411, "float16", False), (1200, 8203, "float32", False),
           (1368, 16384, "bfloat16", False), (912, 25601, "bfloat16", True), (1200, 26001, "float16", True),
           (1300, 12803, "float32", True), (1163, 50001, "bfloat16", True)]


@pytest.mark.parametrize("rows,vocab,dtype,tail", STAYING)
@pytest.mark.parametrize("top,pad,offset", [(24, 0, 0), (100, 3, 5), (1, 8, 8)])
def test_rows_in_turn(gpu_lib, rows, vocab, dtype, tail, top, pad, offset):
    """Rows whose logits or lists are special, in every turn of a CTA, among others that are not; against the reference, and
    all of them against what they give a few at a time, by other kernels."""
    import torch
    x, index, t = case(rows + top, rows, vocab, dtype, top, pad, offset)
    low, inf = torch.finfo(x.dtype).min, float("inf")
    at = [b + k for b in (0, 456, 912) for k in (3, 20, 200, 443) if b + k + 12 < rows]
    for r in at:
        x[r] = -inf
        x[r + 1, 17] = float("nan")
        x[r + 2, vocab - 1] = inf
        x[r + 3] = low
        x[r + 4] = -inf
        x[r + 4, int(index[r + 4, 0].clamp(min=0))] = 1.0
        index[r + 5, 0] = vocab
        index[r + 6] = -1
        index[r + 7] = index[r + 7, :1].clamp(min=0)             # one symbol throughout
        t[r + 7] = -0.7 - float(np.log(top))
        index[r + 8, 0], t[r + 8, 0] = 3, float("nan")
        x[r + 9] = 0.0
        x[r + 10, : vocab - 1] = -inf
        x[r + 11, ::2] = low
    T = 1.5
    r = gpu_lib.mca_distill(x, index, t, T, tail=tail)
    parts = [gpu_lib.mca_distill(x[k:k + 97], index[k:k + 97], t[k:k + 97], T, tail=tail) for k in range(0, rows, 97)]
    for name in ("loss", "lse") + (("rest",) if tail else ()):
        a, b = getattr(r, name), torch.cat([getattr(p, name) for p in parts])
        fine = torch.isfinite(b)
        assert torch.equal(a[~fine].nan_to_num(7.0), b[~fine].nan_to_num(7.0))
        # two evaluations, each within what a few hundred additions of 2^-24 leave
        assert float((a[fine] - b[fine]).abs().div(1 + b[fine].abs()).max()) <= 2e-5
    pick = sorted({q + k for q in at[::4] for k in range(12)} | {0, 1, 300, rows - 2, rows - 1})
    check_picked(gpu_lib, x, index, t, T, tail, torch.tensor(pick, device="cuda"), dtype, r)


@pytest.mark.parametrize("rows,vocab,dtype,tail", STAYING)
def test_rows_in_turn_same_symbols(gpu_lib, rows, vocab, dtype, tail):
    """Lists of 70 that hold symbols twice and more often, beside one another and far apart, all in one piece of 16 bytes, at
    both ends of the row, and taken out by -inf."""
    import torch
    x, index, t = case(vocab, rows, vocab, dtype, 70, 1, 1)
    t = torch.log_softmax(torch.randn(t.shape, device="cuda"), 1) - 1.0
    every = torch.arange(rows, device="cuda")
    index[index < 0] = 11
    index[every % 5 == 0, 1] = index[every % 5 == 0, 0]
    index[every % 5 == 1, 69] = index[every % 5 == 1, 2]
    index[every % 5 == 2, 40] = index[every % 5 == 2, 3]
    index[every % 5 == 3] = torch.arange(70, dtype=torch.int32, device="cuda") + vocab - 70
    index[every % 5 == 4] = torch.arange(70, dtype=torch.int32, device="cuda") % 9
    out_of = every % 10 == 2
    x[out_of, index[out_of, 1].long()] = float("-inf")
    pick = torch.cat([every[:11], every[450:461], every[-6:]])
    check_picked(gpu_lib, x, index, t, 1.0, tail, pick, dtype)


@pytest.mark.parametrize("T", [2.0 ** -20, 0.01, 30.0, 2.0 ** 20])
@pytest.mark.parametrize("rows,vocab,dtype,tail", STAYING[1:3] + STAYING[5:7])
def test_rows_in_turn_at_the_ends_of_temperature(gpu_lib, rows, vocab, dtype, tail, T):
    import torch
    T = float(np.float32(T))
    x, index, t = case(3, rows, vocab, dtype, 20)
    check_picked(gpu_lib, x, index, t, T, tail, torch.arange(0, rows, rows // 12, device="cuda"), dtype)


@pytest.mark.parametrize("rows,vocab,dtype,tail", STAYING)
def test_rows_in_turn_nothing_left_but_the_list(gpu_lib, rows, vocab, dtype, tail):
    """Rows of which nothing but listed symbols is left, by -inf and by the type's lowest value, and some by both."""
    import torch
    x, index, t = case(4, rows, vocab, dtype, 9)
    index[index < 0] = 5
    z = x.gather(1, index.long())
    low = torch.finfo(x.dtype).min
    x.fill_(float("-inf"))
    x[1::3] = low
    x[2::3, : vocab // 2] = low
    x.scatter_(1, index.long(), z)
    t = torch.log_softmax(torch.randn(rows, 10, device="cuda"), 1)[:, :9].contiguous()
    check_picked(gpu_lib, x, index, t, 1.0, tail, torch.arange(0, rows, rows // 14, device="cuda"), dtype)


@pytest.mark.parametrize("rows,vocab,dtype,tail",
                         STAYING + [(70000, 40, "bfloat16", True), (5000, 504, "bfloat16", False),
                                    (3000, 2104, "bfloat16", True), (700, 20000, "bfloat16", True)])
def test_same_bits_wherever_a_row_stands(gpu_lib, rows, vocab, dtype, tail):
    """Rows in another order give their results in that order, bit for bit, and again."""
    import torch
    pad = -vocab % 8                                             # rows that all lie alike
    x, index, t = case(5, rows, vocab, dtype, 12, pad)
    order = torch.randperm(rows, generator=torch.Generator().manual_seed(1)).cuda()
    y = torch.full((rows, vocab + pad), 1.0, dtype=x.dtype, device="cuda")[:, :vocab]
    y.copy_(x[order])
    a = gpu_lib.mca_distill(x, index, t, tail=tail)
    b = gpu_lib.mca_distill(y, index[order].contiguous(), t[order].contiguous(), tail=tail)
    again = gpu_lib.mca_distill(x, index, t, tail=tail)
    one = torch.ones(rows, device="cuda")
    da = gpu_lib.mca_distill_backward(x, index, t, a.lse, one, rest=a.rest)
    db = gpu_lib.mca_distill_backward(y, index[order].contiguous(), t[order].contiguous(), b.lse, one, rest=b.rest)
    assert bool(torch.isfinite(a.loss).all())
    for p, q, s in zip(a, b, again):
        assert p is None or (torch.equal(p[order], q) and torch.equal(p, s))
    assert torch.equal(da[order], db)


CAPTURED = [(912, 16411), (1200, 26001)]


@pytest.mark.parametrize("rows,vocab", CAPTURED)
def test_rows_in_turn_captured(gpu_lib, rows, vocab):
    """Captured on a stream of its own and replayed on new logits and lists, beside an eager call on another stream: the
    eager results, bit for bit."""
    import torch
    zs = [case(s, rows, vocab, "bfloat16", 20) for s in (6, 7)]
    want = [[gpu_lib.mca_distill(*z, 1.5, tail=tail) for tail in (False, True)] for z in zs]
    buf = [a.clone() for a in zs[0]]
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = [gpu_lib.mca_distill(*buf, 1.5, tail=tail, stream=side) for tail in (False, True)]
        torch.cuda.current_stream().wait_stream(side)
    for k in (1, 0, 1):
        for a, b in zip(buf, zs[k]):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(other):
            eager = [gpu_lib.mca_distill(*zs[1 - k], 1.5, tail=tail) for tail in (False, True)]
        torch.cuda.synchronize()
        for mine, ref in ((got, want[k]), (eager, want[1 - k])):
            for p, q in zip(mine, ref):
                assert all(a is None or torch.equal(a, b) for a, b in zip(p, q))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,vocab", [(3000, 300), (3000, 1001), (700, 4001), (930, 20003), (5, 100001)])
def test_gradient_in_place_of_many_rows(gpu_lib, dtype, rows, vocab):
    """Over the logits themselves, a hundred listed symbols in every part of the row: what it is beside them, bit for bit."""
    import torch
    x, index, t = case(vocab, rows, vocab, dtype, 100, 3, 1)
    for tail in (False, True):
        y = torch.empty(rows, vocab + 3, dtype=x.dtype, device="cuda")[:, :vocab]
        y.copy_(x)
        r = gpu_lib.mca_distill(y, index, t, tail=tail)
        g = torch.linspace(-1.0, 2.0, rows, device="cuda")
        out = torch.empty_strided(y.shape, y.stride(), dtype=y.dtype, device="cuda")
        want = gpu_lib.mca_distill_backward(y, index, t, r.lse, g, rest=r.rest, out=out).clone()
        assert gpu_lib.mca_distill_backward(y, index, t, r.lse, g, rest=r.rest, out=y) is y
        assert torch.equal(y, want)
