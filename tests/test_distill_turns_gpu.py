"""The loss against a teacher's list of many rows that are long, or of the lengths at which another kernel takes over
(needs a GPU)."""
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


@pytest.mark.parametrize("rows,vocab,dtype", [(1300, 16380, "bfloat16"), (1300, 16383, "float16"), (1300, 8190, "float32"),
                                              (2500, 16378, "bfloat16"), (2500, 8191, "float32")])
def test_rows_too_long_for_shared_memory_and_too_short_to_stay(gpu_lib, rows, vocab, dtype):
    import torch
    x, index, t = case(vocab, rows, vocab, dtype, 24, 1, 1)
    x[8] = float("-inf")
    x[9, vocab - 1] = float("nan")
    x[10, : vocab - 2] = float("-inf")
    check_picked(gpu_lib, x, index, t, 1.0, False, torch.tensor([0, 1, 8, 9, 10, 1299, rows - 1], device="cuda"), dtype)
