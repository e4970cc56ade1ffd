"""Draws where the steps of the integer sums show: weights around and below half a step, rows whose largest logit comes
late, many rounds to a warp, the largest vocabularies (needs a GPU).

How far a sum may be off. A weight is evaluated to 2^-33 of itself, and rounded to a multiple of 2^-43 of a power of two R that is
at most 2^1.5 times the row's largest weight: half a step for each symbol. Where a larger logit raises R, what a lane has
added up is rounded down to new steps, each time half of what was lost before: 2 steps for each lane, whose pieces have 4
symbols at least, so half a step for each symbol. In all vocab steps of 2^-41.5 of the largest weight, or half as many again
where a symbol is looked for among weights that are rounded anew. The cumulative sum and u times the whole sum may
each be off by that: 2.5 vocab 2^-41.5 < vocab 2^-40."""
import numpy as np
import pytest

import drafts_reference as R
from test_answers_gpu import DT, f64, to_gpu
from test_draw_gpu import check_sample, drafts_case, gpu, uniform

pytestmark = pytest.mark.gpu


def check_within(x, u, r, e=None):
    """Tokens of equal or different rows x [rows or 1, vocab] float64: of positive weight, and none whose part of the
    cumulative sum does not come as near to u times all weights as the sums may be off; log probabilities to match."""
    tok, lp, lse = r.token.cpu().numpy(), f64(r.logprob), f64(r.lse)
    sums = [(v, v.max(), np.exp(v - v.max()), np.cumsum(np.exp(v - v.max()))) for v in x]
    for i in range(len(u)):
        v, m, w, c = sums[i % len(x)]
        t, k = float(u[i]) * c[-1], tok[i]
        off = 2.0 ** -32 * c[-1] + len(v) * 2.0 ** -40 if e is None else e
        assert k >= 0 and w[k] > 0, (i, k)
        assert c[k] > t - off and c[k] - w[k] <= t + off, (i, k, c[k] - t)
        # (a sum that is off by `off` moves its logarithm by that over the sum, which is 1 at least; a rounding to fp32 each)
        want = m + np.log(c[-1])
        assert abs(lse[i] - want) <= 2.0 ** -24 * abs(want) + 1.01 * off / c[-1]
        assert abs(lp[i] - (v[k] - want)) <= 2.0 ** -24 * abs(v[k] - want) + 1.01 * off / c[-1]


# rows and pieces of 16 bytes a row: one, two, four and eight warps to a row, and clusters; 256 pieces to each warp
SHAPES = [(3700, 256), (1900, 512), (1000, 1024), (300, 2048), (50, 16384)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,pieces", SHAPES)
@pytest.mark.parametrize("level", [-29.95, -29.0, -31.5])
def test_a_plateau_before_the_largest_logit(gpu_lib, dtype, rows, pieces, level):
    """Symbols that count while the scale is fine, and each less than half a step when the last logit has raised it: a
    number within their part of the sum draws one of them, or a neighbour, never none."""
    n = 4 if dtype == "float32" else 8
    x = np.full((1, pieces * n), -np.inf)
    x[0, 0] = np.log(2.0 ** -20)
    x[0, 32 * n: 64 * n] = level                                 # a warp's second round, which has its sum kept
    x[0, 64 * n] = 0.0
    xs = to_gpu(x, dtype)
    c = np.cumsum(np.exp(f64(xs)[0]))
    lo, hi = c[0] / c[-1], c[64 * n - 1] / c[-1]
    u = (lo + (hi - lo) * np.linspace(-0.2, 1.2, rows)).astype(np.float32)
    r = gpu_lib.mca_sample_tokens(xs.repeat(rows, 1), gpu(u))
    check_within(f64(xs), u, r)


def test_a_number_at_a_plateau(gpu_lib):
    """The symbol of a number that lies among 128 symbols of 1e-13 each: by the definition where the steps have none left."""
    import torch
    x = torch.full((1, 1024), float("-inf"), device="cuda")
    x[0, 0], x[0, 128:256], x[0, 256] = -3.674689292907715, -29.95, 0.0
    tok = gpu_lib.mca_sample_tokens(x.repeat(3700, 1), torch.full((3700,), 0.024730192497372627, device="cuda")).token
    assert bool((tok == 134).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,pieces", SHAPES)
def test_rising_rows(gpu_lib, dtype, rows, pieces):
    """Logits that rise along the row, by which the scale is raised again and again, and numbers in the part of the small
    weights as well as anywhere."""
    n = 4 if dtype == "float32" else 8
    rng = np.random.default_rng(pieces)
    vocab = pieces * n
    few = 8
    x = np.linspace(-45.0, 0.0, vocab) * rng.uniform(0.3, 1.0, (few, 1)) + 0.5 * rng.standard_normal((few, vocab))
    xs = to_gpu(x, dtype)
    u = np.where(rng.random(rows) < 0.5, rng.random(rows), 2.0 ** rng.uniform(-23.9, 0, rows)).astype(np.float32)
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    r = gpu_lib.mca_sample_tokens(xs.repeat(-(-rows // few), 1)[:rows], gpu(u))
    check_within(f64(xs), u, r)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,vocab", [(3700, 9001), (1900, 20001), (1000, 30011), (3650, 4096)])
def test_many_rounds_to_a_warp(gpu_lib, dtype, rows, vocab):
    """One, two and four warps a row with several groups of rounds each."""
    rng = np.random.default_rng(vocab)
    x = (2.0 * rng.standard_normal((40, vocab)))[rng.integers(0, 40, rows)]
    x[:, ::7] += rng.standard_normal((rows, 1))                  # (other weights in each row)
    check_sample(gpu_lib, to_gpu(x, dtype), uniform(rng, rows))


@pytest.mark.parametrize("rows", [50, 300, 1000, 1900, 3700])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_equal_weights_far_below(gpu_lib, rows, dtype):
    """One logit and thousands of equal ones around half a step of it, which together may be off by half a step each."""
    vocab = 20000
    x = np.full((3, vocab), 0.0)
    x[:, 1:] = np.array([[-30.6], [-29.0], [-27.5]])
    xs = to_gpu(x, dtype)
    rng = np.random.default_rng(rows)
    u = uniform(rng, rows)
    u[::2] = 1 - 2.0 ** -24 * rng.integers(1, 4, len(u[::2]))
    r = gpu_lib.mca_sample_tokens(xs.repeat(-(-rows // 3), 1)[:rows], gpu(u))
    check_within(f64(xs), u, r)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("seqs,vocab", [(3, 20000), (300, 4000), (2000, 2000)])
def test_verify_many_equal_weights_far_below(gpu_lib, dtype, seqs, vocab):
    """The same where a draft was not kept: weights of both nets, each rounded to 2^-43 of the target's sum (half a step each),
    in the cumulative sum and in u times the whole: vocab 2^-42, and 2^-32 of both sums."""
    import torch
    rng = np.random.default_rng(seqs)
    x = np.full((1, vocab), -29.2)
    y = np.full((1, vocab), -30.1)
    x[0, [0, 1, vocab - 1]], y[0, [0, 1, vocab - 1]] = [-12.0, 0.0, 0.3], [-13.0, 0.9, -0.4]
    xs, ys = to_gpu(x, dtype), to_gpu(y, dtype)
    tl, dl = (torch.logsumexp(t.double(), 1).float() for t in (xs, ys))
    p, q = np.exp(f64(xs)[0] - float(tl)), np.exp(f64(ys)[0] - float(dl))
    w = np.clip(p - q, 0, None)
    c = np.cumsum(w)
    u = np.stack([np.full(seqs, 3.0), rng.random(seqs)], 1)
    u[::2, 1] = (c[0] + (c[-2] - c[0]) * np.linspace(-0.2, 1.2, len(u[::2]))) / c[-1]
    u = u.astype(np.float32)
    u[:, 1] = np.minimum(u[:, 1], np.float32(1 - 2.0 ** -24))
    r = gpu_lib.mca_verify_drafts(xs.expand(seqs, 2, vocab).contiguous(), tl.view(1, 1).repeat(seqs, 2),
                                  ys.view(1, 1, vocab).repeat(seqs, 1, 1), dl.view(1, 1).repeat(seqs, 1),
                                  gpu(np.ones((seqs, 1), np.int32)), gpu(u))
    assert int(r.accepted.abs().sum()) == 0
    e = 2.0 ** -32 * (p.sum() + q.sum()) + vocab * 2.0 ** -42
    tok = r.tokens[:, 0].cpu().numpy()
    t = u[:, 1].astype(np.float64) * c[-1]
    assert (tok >= 0).all() and (w[tok] > 0).all()
    assert (c[tok] > t - e).all() and (c[tok] - w[tok] <= t + e).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [(1 << 19) - 1, 1 << 19, (1 << 19) + 1, 700001])
def test_largest_vocabularies(gpu_lib, dtype, vocab):
    """Up to 2^19 symbols by integer sums, and beyond by 64-bit ones."""
    rng = np.random.default_rng(vocab)
    check_sample(gpu_lib, to_gpu(1.5 * rng.standard_normal((3, vocab)), dtype), uniform(rng, 3))


def test_equal_logits_of_the_largest_vocabulary(gpu_lib):
    """The largest sums: 2^19 equal weights, and u on the borders."""
    import torch
    vocab = 1 << 19
    for z in (0.0, 0.34, -0.4):                                  # about one half, and either end, of a power of two
        v = np.unique(np.linspace(0, vocab - 1, 9).astype(int))
        u = (v / vocab).astype(np.float32)
        x = torch.full((len(v), vocab), z, device="cuda")
        r = gpu_lib.mca_sample_tokens(x, gpu(u))
        assert np.array_equal(r.token.cpu().numpy(), v)
        assert float((r.lse.double() - (float(np.float32(z)) + np.log(vocab))).abs().max()) <= 2.0 ** -20


def test_verify_largest_vocabularies(gpu_lib):
    rng = np.random.default_rng(5)
    for vocab in (1 << 19, 600001):
        case = drafts_case(rng, 3, 1, vocab, "float32", near=1.0)
        target, tl, draft, dl, tokens, u = case
        u[1:, 0] = 3.0                                           # never kept
        out, acc, lps, near = R.verify(f64(target), f64(tl), f64(draft), f64(dl), tokens, u, None)
        r = gpu_lib.mca_verify_drafts(target, tl, draft, dl, gpu(tokens), gpu(u))
        assert np.array_equal(r.accepted.cpu().numpy(), acc)
        assert np.array_equal(r.tokens.cpu().numpy()[~near], out[~near])
