"""The answers' operators against their plain 64-bit forms (needs a GPU): quantised rows and integer sums exactly,
the rest within the roundings that answers_reference.py counts."""
import numpy as np
import pytest

import answers_reference as R

pytestmark = pytest.mark.gpu

DT = ["float32", "float16", "bfloat16"]


def torch_dtype(name):
    import torch
    return getattr(torch, name)


def to_gpu(x, dtype="float32", ld=None, offset=0):
    """x [rows, cols] as a CUDA matrix with row distance ld, `offset` elements into its storage, the
    storage around it NaN (or 77 for codes)."""
    import torch
    x = torch.as_tensor(x)
    rows, cols = x.shape
    ld = ld or cols
    t = torch.int8 if x.dtype == torch.int8 else torch_dtype(dtype)
    buf = torch.full((offset + rows * ld + 32,), 77 if t == torch.int8 else float("nan"), dtype=t,
                     device="cuda")
    m = buf.as_strided((rows, cols), (ld, 1), offset)
    m.copy_(x.to(t))
    return m


def f64(t):
    return t.double().cpu().numpy()


def guarded(rows, cols, dtype, ld, offset):
    """An output matrix inside a buffer of a marker; check() that only the matrix was written."""
    import torch
    mark = 77
    buf = torch.full((offset + rows * ld + 64,), mark, dtype=dtype, device="cuda")
    m = buf.as_strided((rows, cols), (ld, 1), offset)

    def check():
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep.as_strided((rows, cols), (ld, 1), offset).fill_(False)
        assert bool((buf[keep] == mark).all())
    return m, check


# ------------------------------------------------------------------------------------------------
# quantised rows
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols,pad,offset", [
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 15, 0, 1), (4, 16, 0, 0), (7, 17, 3, 5), (2, 127, 0, 0),
    (9, 391, 0, 3), (6, 784, 0, 0), (3, 1024, 8, 8), (2, 4096, 0, 0), (3, 4097, 0, 1),
    (2, 16384, 0, 0), (1, 40003, 0, 0), (300, 64, 0, 0), (2000, 33, 1, 0)])
def test_quantize_rows(gpu_lib, dtype, rows, cols, pad, offset):
    import torch
    rng = np.random.default_rng(rows * 100003 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1)))
    if rows > 2:
        x[1] = 0.0
    xg = to_gpu(x, dtype, cols + pad, offset)
    codes, check = guarded(rows, cols, torch.int8, cols + pad, offset)
    scale = torch.empty(rows, device="cuda")
    gpu_lib.mca_quantize_rows(xg, codes, scale)
    q, s = R.quantize(f64(xg))
    assert np.array_equal(scale.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), q)
    check()
    c2, s2 = gpu_lib.mca_quantize_rows(xg)
    assert torch.equal(c2, codes) and torch.equal(s2, scale)
    assert c2.stride(0) % 16 == 0 or rows == 1


def test_quantize_halves_and_borders(gpu_lib):
    """Quotients at and next to a half: the row's largest magnitude is 127 s, the others (n + 1/2) s and their
    neighbours in fp32, for scales that are not powers of two."""
    import torch
    rows = []
    for s in (1.0, 0.1, 3.7, 1e-3, 0.0123457, 2.0 ** -120, 1e30):
        s = np.float32(s)
        top = np.float32(127.0) * s
        s = top / np.float32(127.0)
        h = ((np.arange(127) + 0.5) * np.float64(s)).astype(np.float32)
        rows.append(np.concatenate([[top], h, np.nextafter(h, np.float32(np.inf)),
                                    np.nextafter(h, np.float32(0)), -h, -np.nextafter(h, np.float32(0))]))
    x = np.stack(rows).astype(np.float64)
    codes, scale = gpu_lib.mca_quantize_rows(to_gpu(x))
    q, s = R.quantize(x)
    assert np.array_equal(scale.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), q)


@pytest.mark.parametrize("cols", [5, 200, 3000, 20000])
def test_quantize_special_rows(gpu_lib, cols):
    """Zeros, subnormal and largest values, infinities and NaN; other rows as if these were not there."""
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((10, cols)).astype(np.float32)
    x[1] = 0.0
    x[2] = -0.0
    x[3, cols - 1] = np.nan
    x[4, 0] = np.inf
    x[5, cols // 2] = -np.inf
    x[6] = (rng.integers(-40, 41, cols) * 2.0 ** -149).astype(np.float32)     # scale rounds to 0
    x[7] = (rng.integers(-5000, 5001, cols) * 2.0 ** -149).astype(np.float32)  # scale is subnormal
    x[8] = np.finfo(np.float32).max
    x[9] *= np.float32(1e-36)
    codes, scale = gpu_lib.mca_quantize_rows(to_gpu(x))
    q, s = R.quantize(x.astype(np.float64))
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), q)


# ------------------------------------------------------------------------------------------------
# layers on codes
# ------------------------------------------------------------------------------------------------

def linear_case(rng, rows, n_in, n_out, ternary=False):
    xq = rng.integers(-127, 128, (rows, n_in)).astype(np.int8)
    wq = (rng.integers(-1, 2, (n_out, n_in)) if ternary
          else rng.integers(-127, 128, (n_out, n_in))).astype(np.int8)
    xs = np.exp(rng.standard_normal(rows)).astype(np.float32) / 127
    ws = (np.exp(rng.standard_normal(n_out)) / (73.0 * np.sqrt(n_in) * (1 if ternary else 60))
          ).astype(np.float32)
    return xq, wq, xs, ws


def gpu_vec(v):
    import torch
    return None if v is None else torch.from_numpy(v).cuda()


def run_linear(gpu_lib, xq, wq, xs, ws, bias, act, g, dtype, ldx=None, ldw=None, pad=0, off=(0, 0, 0)):
    rows, n_out = xq.shape[0], wq.shape[0]
    y, check = guarded(rows, n_out, torch_dtype(dtype), n_out + pad, off[2])
    gpu_lib.mca_code_linear(to_gpu(xq, ld=ldx, offset=off[0]), gpu_vec(xs),
                            to_gpu(wq, ld=ldw, offset=off[1]), gpu_vec(ws), bias=gpu_vec(bias),
                            act=act, act_param=g, out=y)
    check()
    return f64(y)


def check_linear(gpu_lib, rng, rows, n_in, n_out, dtype="float32", act="identity", g=0.0, bias=False,
                 ternary=False, **kw):
    xq, wq, xs, ws = linear_case(rng, rows, n_in, n_out, ternary)
    b = rng.standard_normal(n_out).astype(np.float32) if bias else None
    got = run_linear(gpu_lib, xq, wq, xs, ws, b, act, g, dtype, **kw)
    want, tol = R.code_linear(xq, xs, wq, ws, b, act, g, dtype)
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("rows", [1, 2, 3, 7, 8, 9, 16, 17, 33, 64, 65, 128, 129, 200, 257, 700])
@pytest.mark.parametrize("n_in,n_out", [(1, 1), (16, 5), (64, 64), (65, 130), (127, 10), (256, 256),
                                        (784, 300), (1040, 129)])
def test_code_linear_sizes(gpu_lib, rows, n_in, n_out):
    check_linear(gpu_lib, np.random.default_rng(rows * 7919 + n_in), rows, n_in, n_out)


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 4096, 16384), (4, 16384, 100), (20, 9000, 1001),
                                             (48, 4096, 4096), (300, 4096, 520), (1000, 2100, 257),
                                             (2347, 391, 1001), (513, 131071, 3)])
@pytest.mark.parametrize("dtype", DT)
def test_code_linear_larger(gpu_lib, rows, n_in, n_out, dtype):
    check_linear(gpu_lib, np.random.default_rng(rows), rows, n_in, n_out, dtype, bias=True)


@pytest.mark.parametrize("act,g", [("identity", 0.0), ("tanh", 0.0), ("sigmoid", 0.0), ("relu", 0.0),
                                   ("gaussian", 1.0), ("gaussian", 0.4), ("gelu", 0.0)])
@pytest.mark.parametrize("rows", [3, 30, 600])
@pytest.mark.parametrize("dtype", DT)
def test_code_linear_transfer_functions(gpu_lib, act, g, rows, dtype):
    check_linear(gpu_lib, np.random.default_rng(rows), rows, 200, 150, dtype, act, g, bias=rows != 30,
                 ternary=rows == 30)


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
@pytest.mark.parametrize("n_in,kw", [
    (64, dict(ldx=80, ldw=96)), (64, dict(off=(16, 32, 0))), (64, dict(off=(1, 0, 3))),
    (64, dict(off=(0, 7, 0), pad=5)), (64, dict(ldx=65)), (64, dict(ldw=71)), (100, dict(ldx=112)),
    (100, dict(ldx=112, ldw=112)), (1000, dict(ldw=1008, pad=1)), (33, dict(pad=7, off=(3, 5, 1)))])
def test_code_linear_strides_and_alignment(gpu_lib, rows, n_in, kw):
    """Rows on and off 16-byte boundaries; what lies between them is not read into the sums (it is 77)."""
    check_linear(gpu_lib, np.random.default_rng(rows + n_in), rows, n_in, 130, **kw)


@pytest.mark.parametrize("rows", [1, 9, 70, 260])
@pytest.mark.parametrize("n_in", [1024, 1040, 2048, 5000])
@pytest.mark.parametrize("code", [-128, -127, 127])
def test_code_linear_largest_sums(gpu_lib, rows, n_in, code):
    """Sums beyond 2^24, of codes of one sign, are exact integers: scales of 1 show their rounding to fp32
    and nothing else. An odd sum of its own in every output."""
    n_out = 150
    rng = np.random.default_rng(n_in)
    xq = np.full((rows, n_in), code, np.int8)
    wq = np.full((n_out, n_in), code, np.int8)
    wq[:, 0] = rng.integers(-128, 128, n_out)
    xq[:, 1] = rng.integers(-128, 128, rows)
    xq[:, 0] = 1
    got = run_linear(gpu_lib, xq, wq, np.ones(rows, np.float32), np.ones(n_out, np.float32), None,
                     "identity", 0.0, "float32")
    s = xq.astype(np.int64) @ wq.astype(np.int64).T
    assert np.array_equal(got, s.astype(np.float32).astype(np.float64))


def sums_on_gpu(xq, wq):
    """Integer sums in fp64, which holds them exactly."""
    return (xq.double() @ wq.double().T)


@pytest.mark.parametrize("dtype,act,g,bias", [("float32", "identity", 0.0, False),
                                              ("float16", "gaussian", 1.0, False),
                                              ("bfloat16", "gelu", 0.0, True),
                                              ("float32", "tanh", 0.0, True)])
@pytest.mark.parametrize("rows,n_in,n_out,off,pad", [
    # tiles of the pair kernel: whole, ragged, of one to six exact sums, rows off 16-byte boundaries
    (2048, 1024, 2048, (0, 0, 0), 0), (2491, 432, 5121, (0, 0, 0), 3), (5901, 176, 2687, (1, 0, 1), 0),
    (700, 2992, 4000, (0, 7, 0), 0), (1501, 5001, 3003, (0, 0, 3), 1), (3086, 64, 10970, (0, 0, 0), 0),
    # of the cluster kernel, up to 128 samples and more
    (57, 4880, 6140, (0, 0, 0), 0), (36, 11808, 1660, (5, 0, 0), 0), (105, 4992, 3096, (0, 0, 1), 2),
    (128, 3001, 500, (0, 3, 0), 0), (300, 8192, 700, (0, 0, 0), 0), (65, 131071, 129, (0, 0, 0), 0)])
def test_code_linear_many(gpu_lib, rows, n_in, n_out, off, pad, dtype, act, g, bias):
    """Sizes beyond the numpy form: its formula on sums that the GPU makes in fp64, from codes of one sign
    and of both."""
    import torch
    rng = np.random.default_rng(rows + n_in)
    xq, wq, xs, ws = linear_case(rng, rows, n_in, n_out)
    xq[: rows // 2] = np.abs(xq[: rows // 2])
    wq[: n_out // 2] = np.abs(wq[: n_out // 2])
    b = rng.standard_normal(n_out).astype(np.float32) if bias else None
    got = run_linear(gpu_lib, xq, wq, xs, ws, b, act, g, dtype, off=off, pad=pad)
    s = sums_on_gpu(torch.from_numpy(xq).cuda(), torch.from_numpy(wq).cuda()).cpu().numpy()
    if act == "identity" and b is None:
        want = (s.astype(np.float32) * xs[:, None]) * ws
        assert np.array_equal(got, want.astype(np.float64))
        return
    want, tol = R.code_fields(s, xs, ws, b, act, g, dtype)
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("rows,n_in,n_out", [(2048, 1040, 2048), (1500, 5000, 3000), (100, 9000, 600)])
@pytest.mark.parametrize("code", [-128, 127])
def test_code_linear_largest_sums_of_many(gpu_lib, rows, n_in, n_out, code):
    import torch
    rng = np.random.default_rng(n_in)
    xq = np.full((rows, n_in), code, np.int8)
    wq = np.full((n_out, n_in), code, np.int8)
    wq[:, 0] = rng.integers(-128, 128, n_out)
    xq[:, 1] = rng.integers(-128, 128, rows)
    xq[:, 0] = 1
    got = run_linear(gpu_lib, xq, wq, np.ones(rows, np.float32), np.ones(n_out, np.float32), None,
                     "identity", 0.0, "float32")
    s = sums_on_gpu(torch.from_numpy(xq).cuda(), torch.from_numpy(wq).cuda()).cpu().numpy()
    assert np.array_equal(got, s.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("rows,n_out", [(7, 3001), (2500, 2), (40001, 45), (3001, 300)])
@pytest.mark.parametrize("dtype", DT)
def test_gelu_of_any_field(gpu_lib, rows, n_out, dtype):
    """Fields over the whole range, which are the scales' products exactly, so that only the function is off: 18 + 1.5 z^2
    half steps at most (the exponent's roundings grow with its size), tails below 2^-126 flushed."""
    import torch
    rng = np.random.default_rng(rows)
    xs = np.concatenate([[0.0, 1e-30, 3e4, np.nan, np.inf], rng.uniform(0, 14, rows)])[:rows].astype(np.float32)
    ws = np.concatenate([[1.0, -1.0], rng.uniform(-1, 1, n_out)])[:n_out].astype(np.float32)
    with np.errstate(all="ignore"):
        z = (xs[:, None] * ws).astype(np.float32).astype(np.float64)
    one = np.ones((rows, 1), np.int8), np.ones((n_out, 1), np.int8)
    got = run_linear(gpu_lib, *one, xs, ws, None, "gelu", 0.0, dtype)
    assert np.isnan(got[np.isnan(z)]).all() and (got[z == np.inf] == np.inf).all() and (got[z == -np.inf] == 0).all()
    fin = np.isfinite(z)
    z, got = z[fin], got[fin]
    want = R.act("gelu", z, 0.0)[0]
    tol = 1.01 * R.U * (18 + 1.5 * np.minimum(z * z, 400.0)) * np.abs(want) + 20 * 2.0 ** -126
    if dtype != "float32":
        tol = tol + R.HALF_STEP[dtype] * (np.abs(want) + tol) + R.TINY[dtype]
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())
    assert dtype == "float32" or torch.finfo(torch_dtype(dtype)).max > np.abs(want).max()


def test_code_linear_scales(gpu_lib):
    """Scales of zero, tiny and huge magnitude, infinities and NaN go through by IEEE rules."""
    rng = np.random.default_rng(3)
    for rows in (4, 40, 400):
        xq, wq, xs, ws = linear_case(rng, rows, 96, 70)
        xs[:4] = [0.0, 1e-30, 1e30, np.nan]
        ws[:4] = [1e-30, 0.0, 1e30, np.inf]
        with np.errstate(all="ignore"):
            s = (xq.astype(np.int64) @ wq.astype(np.int64).T).astype(np.float32)
            for dtype in DT:
                got = run_linear(gpu_lib, xq, wq, xs, ws, None, "identity", 0.0, dtype)
                want = ((s * xs[:, None]) * ws)
                assert want.dtype == np.float32
                import torch
                want = torch.from_numpy(want).to(torch_dtype(dtype)).double().numpy()
                assert np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------
# log probabilities
# ------------------------------------------------------------------------------------------------

def check_logprobs(gpu_lib, x, targets, top, dtype, ld=None, offset=0):
    import torch
    rows = x.shape[0]
    xg = to_gpu(x, dtype, ld, offset)
    t = None if targets is None else torch.from_numpy(np.asarray(targets, np.int32)).cuda()
    r = gpu_lib.mca_token_logprobs(xg, t, top=top)
    want = R.logprobs(f64(xg), np.full(rows, -1) if targets is None else targets, top)
    for k in ("lse", "entropy") + (() if targets is None else ("logprob",)):
        got, w, tol = f64(getattr(r, k)), want[k], want["tol_" + k]
        fin = np.isfinite(w)
        assert np.array_equal(np.where(fin, 0.0, got), np.where(fin, 0.0, w), equal_nan=True), k
        err = np.abs(got[fin] - w[fin])
        assert np.all(err <= tol[fin]), (k, float((err / np.maximum(tol[fin], 1e-30)).max()))
    assert (r.logprob is None) == (targets is None)
    if top == 0:
        assert r.top_index is None and r.top_logprob is None
        return r
    assert np.array_equal(r.top_index.cpu().numpy(), want["top_index"])
    got, w = f64(r.top_logprob), want["top_logprob"]
    fin = np.isfinite(w)
    assert np.array_equal(np.where(fin, 0.0, got), np.where(fin, 0.0, w), equal_nan=True)
    tol = want["tol_lse"][:, None] + 3 * R.U * (np.abs(w) + np.abs(np.where(fin, w, 0)).max())
    assert np.all(np.abs(got[fin] - w[fin]) <= tol[fin])
    return r


VOCABS = [1, 2, 3, 10, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 511, 513, 1000, 1024, 1025, 2048,
          4097, 8191, 20011, 50001]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprobs_sizes(gpu_lib, vocab, dtype):
    rng = np.random.default_rng(vocab)
    for rows, top, pad, offset in [(1, 0, 0, 0), (3, 1, 3, 1), (37 if vocab < 5000 else 5, 5, 0, 0),
                                   (2, 32, 8, 0), (6, 20, 0, 3)]:
        x = 3 * rng.standard_normal((rows, vocab))
        t = rng.integers(0, vocab, rows)
        if rows > 2:
            t[-1] = -1
        check_logprobs(gpu_lib, x, t, top, dtype, vocab + pad, offset)


@pytest.mark.parametrize("rows,vocab,top", [(1, 128000, 20), (2, 160001, 32), (400, 3001, 8),
                                            (1500, 700, 5), (5000, 65, 5), (20011, 10, 1), (9, 262144, 1),
                                            (1100, 1500, 32), (1031, 8191, 20), (1030, 2049, 1)])
def test_logprobs_many(gpu_lib, rows, vocab, top):
    rng = np.random.default_rng(rows)
    x = (2 * rng.standard_normal((rows, vocab))).astype(np.float32)
    check_logprobs(gpu_lib, x, rng.integers(0, vocab, rows), top, "bfloat16")


@pytest.mark.parametrize("vocab", [1, 7, 40, 300, 1500, 9000, 70001])
@pytest.mark.parametrize("dtype", DT)
def test_logprobs_special_rows(gpu_lib, vocab, dtype):
    """Rows whose mask leaves nothing or one symbol, masks of the type's lowest value, infinities and NaN;
    targets that are masked, absent or out of range."""
    import torch
    rng = np.random.default_rng(vocab)
    low = torch.finfo(torch_dtype(dtype)).min
    x = 3 * rng.standard_normal((16, vocab))
    t = rng.integers(0, vocab, 16)
    x[0] = -np.inf
    x[1] = -np.inf
    x[1, vocab - 1] = 2.0
    x[2] = low
    x[3] = low
    x[3, vocab // 2] = 1.0
    x[4, rng.random(vocab) < 0.5] = -np.inf
    x[5, vocab // 3] = np.nan
    x[6, vocab - 1] = np.inf
    x[7, 0] = np.inf
    x[8] = 0.0
    x[9] = -60000.0 if dtype == "float16" else -1e30
    x[10] = 60000.0 if dtype == "float16" else 1e30
    x[11] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    x[12] *= 300.0
    t[0], t[1] = 0, vocab - 1
    t[4] = int(np.argmin(x[4]))
    t[13], t[14], t[15] = -1, vocab, -2
    t[5] = -1
    check_logprobs(gpu_lib, x, t, 12, dtype)
    check_logprobs(gpu_lib, x, None, 0, dtype)


@pytest.mark.parametrize("vocab", [33, 500, 4000, 30000, 100003])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_alternatives_in_any_order(gpu_lib, vocab, top):
    """The largest logits anywhere: falling and rising rows, all equal, two values, the largest in one stripe of
    neighbours or at one distance, at either end."""
    i = np.arange(vocab)
    rng = np.random.default_rng(vocab + top)
    rows = [-i / 64.0, i / 64.0, np.zeros(vocab), (i % 2).astype(float),
            np.where((i >= vocab // 3) & (i < vocab // 3 + 40), 5.0 + (i % 7), rng.standard_normal(vocab)),
            rng.integers(0, 3, vocab).astype(float), np.where(i >= vocab - 5, 9.0, -i / 100.0)]
    for step in (8, 32, 256, 1024, 2048, 4096):
        rows.append(np.where(i % step == step // 2, 8.0 - i / vocab, 0.0))
    check_logprobs(gpu_lib, np.stack(rows), rng.integers(0, vocab, len(rows)), top, "float32")


@pytest.mark.parametrize("vocab,top", [(1100, 32), (3000, 7), (8000, 32)])
def test_many_rows_in_any_order(gpu_lib, vocab, top):
    """The same rows, and rows whose mask leaves nothing or less than is asked for, among more than a thousand."""
    i = np.arange(vocab)
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((1030, vocab))
    x[0], x[1], x[2], x[3] = -i / 64.0, i / 64.0, 0.0, i % 2
    x[4] = np.where(i % 32 == 16, 8.0 - i / vocab, 0.0)
    x[5] = np.where(i % 256 == 128, 8.0, rng.integers(0, 3, vocab))
    x[6] = -np.inf
    x[7] = np.where(i < 5, 1.0, -np.inf)
    x[8] = np.where(i >= vocab - 5, 1.0, np.finfo(np.float32).min)
    x[9, vocab // 2] = np.nan
    x[10, 0] = np.inf
    x[11] = -1e32
    x[1029] = -i / 64.0
    check_logprobs(gpu_lib, x, rng.integers(0, vocab, 1030), top, "float32")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,vocab,top", [(3, 70001, 32), (170, 9001, 20), (700, 4099, 32), (3000, 1200, 8)])
def test_fewer_symbols_than_alternatives(gpu_lib, rows, vocab, top, dtype):
    """Masks that leave less symbols than are asked for, with -inf, the type's lowest value, both of them, or
    falling values near it behind; at the row's ends, side by side, anywhere."""
    import torch
    rng = np.random.default_rng(rows + top)
    low = float(torch.finfo(torch_dtype(dtype)).min)
    x = rng.standard_normal((rows, vocab))
    for r in range(min(rows, 60)):
        left = rng.choice(vocab, r % (top + 2), replace=False) if r % 3 else np.arange(r % top)
        v = x[r, left]
        x[r] = [-np.inf, low, low][r // 3 % 3]
        if r // 3 % 3 == 2:
            x[r, rng.random(vocab) < 0.9] = -np.inf
        if r % 7 == 6 and dtype != "float16":
            x[r] = -2e36 - 1e33 * (np.arange(vocab) // 3) * rng.choice([-0.01, 1.0])
        x[r, left] = v
    check_logprobs(gpu_lib, x, rng.integers(0, vocab, rows), top, dtype)


def test_logprobs_of_shifted_rows(gpu_lib):
    """A common shift of a row's logits changes neither log probabilities nor entropy: differences are taken
    before exponentials."""
    rng = np.random.default_rng(5)
    base = np.round(64 * rng.standard_normal((6, 4000))) / 64
    x = base + np.array([0.0, 64.0, -64.0, 1024.0, -1024.0, 4096.0])[:, None]
    check_logprobs(gpu_lib, x, rng.integers(0, 4000, 6), 5, "float32")


# ------------------------------------------------------------------------------------------------
# their gradient
# ------------------------------------------------------------------------------------------------

def check_backward(gpu_lib, x, t, gl, ge, dtype, pad=0, offset=0, inplace=False):
    import torch
    rows, vocab = x.shape
    xg = to_gpu(x, dtype, vocab + pad, offset)
    x64 = f64(xg)
    tg = torch.from_numpy(np.asarray(t, np.int32)).cuda()
    r = gpu_lib.mca_token_logprobs(xg, tg)
    lse, ent = f64(r.lse), f64(r.entropy)
    out, check = (xg, lambda: None) if inplace else guarded(rows, vocab, xg.dtype, vocab + pad, offset)
    gpu_lib.mca_token_logprobs_backward(xg, tg if gl is not None else None, r.lse,
                                        r.entropy if ge is not None else None, gpu_vec(gl),
                                        gpu_vec(ge), out=out)
    check()
    want, tol = R.backward(x64, t, lse, ent, gl, ge, dtype)
    got = f64(out)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    assert np.all(np.abs(got - want)[~nan] <= tol[~nan]), \
        float((np.abs(got - want) / tol)[~nan].max())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab", [1, 2, 7, 10, 32, 33, 65, 128, 255, 1000, 1025, 4096, 9001, 50001])
def test_backward_sizes(gpu_lib, vocab, dtype):
    rng = np.random.default_rng(vocab)
    for rows, pad, offset, which, inplace in [(1, 0, 0, 3, False), (5, 3, 1, 3, False),
                                              (4, 0, 0, 1, False), (3, 8, 8, 2, False),
                                              (70 if vocab < 5000 else 6, 0, 0, 3, True)]:
        x = 3 * rng.standard_normal((rows, vocab))
        t = rng.integers(0, vocab, rows)
        if rows > 2:
            t[1] = -1
        gl = rng.standard_normal(rows).astype(np.float32) if which & 1 else None
        ge = rng.standard_normal(rows).astype(np.float32) if which & 2 else None
        check_backward(gpu_lib, x, t, gl, ge, dtype, pad, offset, inplace)


@pytest.mark.parametrize("vocab", [1, 40, 300, 5000, 70001])
@pytest.mark.parametrize("dtype", DT)
def test_backward_special_rows(gpu_lib, vocab, dtype):
    import torch
    rng = np.random.default_rng(vocab)
    x = 3 * rng.standard_normal((10, vocab))
    t = rng.integers(0, vocab, 10)
    x[0] = -np.inf
    x[1] = -np.inf
    x[1, vocab - 1] = 2.0
    x[2] = torch.finfo(torch_dtype(dtype)).min
    x[3, rng.random(vocab) < 0.5] = -np.inf
    x[3, 0] = 0.5
    x[4, vocab // 3] = np.nan
    x[5, vocab - 1] = np.inf
    t[6], t[7], t[8] = -1, vocab, -2
    gl = rng.standard_normal(10).astype(np.float32)
    ge = rng.standard_normal(10).astype(np.float32)
    check_backward(gpu_lib, x, t, gl, ge, dtype)
    check_backward(gpu_lib, x, t, gl, None, dtype)


def test_backward_against_differences(gpu_lib):
    """The gradient against central differences of the 64-bit forms (step h: off by h^2 / 6 times the third
    derivative, which is below 8 for |g| <= 1 and V = 20, and 2^-51 / h of rounding)."""
    rng = np.random.default_rng(11)
    rows, V, h = 4, 20, 1e-4
    x = rng.standard_normal((rows, V)).astype(np.float32).astype(np.float64)
    t = rng.integers(0, V, rows)
    gl = rng.uniform(-1, 1, rows).astype(np.float32)
    ge = rng.uniform(-1, 1, rows).astype(np.float32)
    import torch
    xg, tg = to_gpu(x), torch.from_numpy(t.astype(np.int32)).cuda()
    r = gpu_lib.mca_token_logprobs(xg, tg)
    got = f64(gpu_lib.mca_token_logprobs_backward(xg, tg, r.lse, r.entropy, gpu_vec(gl), gpu_vec(ge)))

    def f(z):
        w = R.logprobs(z, t, 0)
        return gl * w["logprob"] + ge * w["entropy"]
    for v in range(V):
        e = np.zeros(V)
        e[v] = h
        diff = (f(x + e) - f(x - e)) / (2 * h)
        # fp32: a dozen roundings of values below 8
        assert np.all(np.abs(got[:, v] - diff) <= 8 * h * h + 2.0 ** -40 / h * 2.0 ** -8 + 100 * R.U)


# ------------------------------------------------------------------------------------------------
# use: streams, graphs, together
# ------------------------------------------------------------------------------------------------

def answers(gpu_lib, x, w, ws, t, stream=None):
    q, s = gpu_lib.mca_quantize_rows(x, stream=stream)
    y = gpu_lib.mca_code_linear(q, s, w, ws, dtype=x.dtype, stream=stream)
    r = gpu_lib.mca_token_logprobs(y, t, top=4, stream=stream)
    g = gpu_lib.mca_token_logprobs_backward(y, t, r.lse, r.entropy, r.logprob, r.entropy,
                                            stream=stream)
    return [q, s, y, *r, g]


@pytest.mark.parametrize("rows,n_in,vocab,ldw", [(1, 256, 1000, 256), (33, 100, 65, 100),
                                                 (300, 512, 3001, 512), (2000, 512, 3001, 512)])
def test_stream_and_graph(gpu_lib, rows, n_in, vocab, ldw):
    """The chain on another stream, captured and replayed on new inputs: bit for bit the eager results."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, n_in, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    w = torch.randint(-127, 128, (vocab, ldw), generator=g, device="cuda").to(torch.int8)
    ws = torch.rand(vocab, generator=g, device="cuda") * 1e-3
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    x2 = torch.randn(rows, n_in, generator=g, device="cuda").to(torch.bfloat16)
    want, want2 = answers(gpu_lib, x, w, ws, t), answers(gpu_lib, x2, w, ws, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = answers(gpu_lib, x, w, ws, t, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = answers(gpu_lib, x, w, ws, t, stream=side)             # the stream itself
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    buf = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = answers(gpu_lib, buf, w, ws, t)
    for src, ref in ((x2, want2), (x, want)):
        buf.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, ref))


def test_two_graphs_at_once(gpu_lib):
    """Two captured chains replayed at the same time on two streams keep to their own buffers."""
    import torch
    made = []
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(40, 777, generator=g, device="cuda")
        w = torch.randint(-127, 128, (901, 777), generator=g, device="cuda").to(torch.int8)
        ws = torch.rand(901, generator=g, device="cuda") * 1e-3
        t = torch.randint(0, 901, (40,), generator=g, device="cuda", dtype=torch.int32)
        want = answers(gpu_lib, x, w, ws, t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = answers(gpu_lib, x, w, ws, t)
        made.append((graph, res, want, torch.cuda.Stream(), x, w, ws, t))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, _, _, st, *_ in made:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, res, want, *_ in made:
        assert all(torch.equal(a, b) for a, b in zip(res, want))


def test_same_results_again(gpu_lib):
    """No order of arrival changes a result: ten calls agree bit for bit."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    for rows, n_in, vocab in ((1, 4096, 50001), (17, 2048, 4096), (600, 1500, 700), (100, 5000, 3001),
                              (2000, 512, 3001)):
        x = torch.randn(rows, n_in, generator=g, device="cuda")
        w = torch.randint(-127, 128, (vocab, n_in), generator=g, device="cuda").to(torch.int8)
        ws = torch.rand(vocab, generator=g, device="cuda") * 1e-3
        t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        want = answers(gpu_lib, x, w, ws, t)
        for _ in range(10):
            assert all(torch.equal(a, b) for a, b in zip(answers(gpu_lib, x, w, ws, t), want))


def test_offsets_beyond_32_bits(gpu_lib):
    """Rows that lie more than 2^31 elements into their matrix."""
    import torch
    V, rows = 70001, 31001                                   # 2.17e9 logits, 4.3 GB
    x = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    t = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32)
    r = gpu_lib.mca_token_logprobs(x, t, top=3)
    last = slice(rows - 3, rows)
    alone = gpu_lib.mca_token_logprobs(x[last].clone(), t[last].clone(), top=3)
    want = R.logprobs(f64(x[last]), t[last].cpu().numpy(), 3)
    assert np.array_equal(r.top_index[last].cpu().numpy(), want["top_index"])
    for k in ("logprob", "entropy", "lse"):
        a, b = f64(getattr(r, k)[last]), f64(getattr(alone, k))
        assert np.all(np.abs(a - want[k]) <= want["tol_" + k])
        assert np.all(np.abs(b - want[k]) <= want["tol_" + k])
    gl = torch.randn(rows, device="cuda")
    g1 = gpu_lib.mca_token_logprobs_backward(x[last].clone(), t[last].clone(), r.lse[last].clone(),
                                             None, gl[last].clone())
    gpu_lib.mca_token_logprobs_backward(x, t, r.lse, None, gl, out=x)
    assert torch.equal(x[last], g1)
    del x, g1
    q = torch.zeros(rows, V, dtype=torch.int8, device="cuda")
    src = torch.randn(3, V, device="cuda")
    wide = torch.zeros(rows, V, dtype=torch.bfloat16, device="cuda")
    wide[last] = src.to(torch.bfloat16)
    s = torch.empty(rows, device="cuda")
    gpu_lib.mca_quantize_rows(wide, q, s)
    qn, sn = R.quantize(f64(wide[last]))
    assert np.array_equal(q[last].cpu().numpy(), qn) and np.array_equal(s[last].cpu().numpy(), sn)
    assert float(s[:-3].abs().max()) == 0.0


def test_refusals_on_the_device(gpu_lib):
    """Host memory, other dtypes, wrong shapes and strides, overlapping outputs: refused before a launch."""
    import torch
    x = torch.randn(4, 32, device="cuda")
    v4 = torch.zeros(4, device="cuda")
    i8 = torch.zeros(4, 32, dtype=torch.int8, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [lambda: gpu_lib.mca_quantize_rows(x.double()),
           lambda: gpu_lib.mca_quantize_rows(x.t()),
           lambda: gpu_lib.mca_quantize_rows(x, codes=i8[:, :31]),
           lambda: gpu_lib.mca_quantize_rows(x, scale=v4[:3]),
           lambda: gpu_lib.mca_code_linear(i8, v4, i8[:, :16], v4),
           lambda: gpu_lib.mca_code_linear(i8, v4[:2], i8, v4),
           lambda: gpu_lib.mca_code_linear(i8, v4.cpu(), i8, v4),
           lambda: gpu_lib.mca_code_linear(i8, v4, i8, v4, out=x),
           lambda: gpu_lib.mca_code_linear(i8, v4, i8, v4, dtype=torch.float64),
           lambda: gpu_lib.mca_token_logprobs(x, t.long()),
           lambda: gpu_lib.mca_token_logprobs(x, t, top=33),
           lambda: gpu_lib.mca_token_logprobs(x[0], t),
           lambda: gpu_lib.mca_token_logprobs_backward(x, t, v4, v4, v4, out=x[:, :31])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    worse = [lambda: gpu_lib.mca_token_logprobs(x.expand(4, 32)[0:1].expand(4, 32), t),
             lambda: gpu_lib.mca_token_logprobs_backward(x, t, v4, None, None),
             lambda: gpu_lib.mca_token_logprobs_backward(x, t, v4, None, v4, v4)]
    buf = torch.zeros(300, device="cuda")
    a, b = buf.as_strided((4, 32), (32, 1), 0), buf.as_strided((4, 32), (32, 1), 8)
    worse.append(lambda: gpu_lib.mca_token_logprobs_backward(a, t, v4, None, v4, out=b))
    for call in worse:
        with pytest.raises(gpu_lib.MCAError) as e:
            call()
        assert e.value.status == gpu_lib.MCA_ERR_INVALID
    # zero rows: results without elements
    q, s = gpu_lib.mca_quantize_rows(x[:0])
    assert q.shape == (0, 32) and s.shape == (0,)
    assert gpu_lib.mca_code_linear(i8[:0], v4[:0], i8, v4).shape == (0, 4)
    r = gpu_lib.mca_token_logprobs(x[:0], t[:0], top=2)
    assert r.logprob.shape == (0,) and r.top_index.shape == (0, 2)
    assert gpu_lib.mca_token_logprobs_backward(x[:0], t[:0], v4[:0], None, v4[:0]).shape == (0, 32)
