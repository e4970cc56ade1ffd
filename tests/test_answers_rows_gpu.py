"""Log probabilities of many long rows: one, two, four or eight warps per row against the plain 64-bit form, row by row
where the values differ (needs a GPU)."""
import numpy as np
import pytest

import answers_reference as R

pytestmark = pytest.mark.gpu
DT = ["float32", "float16", "bfloat16"]


def rows_of(rng, V, dtype):
    """Rows of every kind that the passes tell apart."""
    import torch
    i = np.arange(V)
    low = float(torch.finfo(getattr(torch, dtype)).min)
    x = [2 * rng.standard_normal(V) for _ in range(6)]
    x += [-i / 64.0, i / 64.0, np.zeros(V), (i % 2).astype(float), rng.integers(0, 3, V).astype(float),
          np.where(i % 32 == 16, 8.0 - i / V, 0.0), np.where(i % 256 == 128, 8.0, rng.integers(0, 3, V)),
          np.where(i >= V - 5, 9.0, -i / 100.0), np.where((i >= V // 3) & (i < V // 3 + 40), 5.0 + i % 7, x[0])]
    m = rng.standard_normal((9, V))
    m[0] = -np.inf
    m[1, i % 97 != 5] = -np.inf
    m[2, i >= 5] = -np.inf
    m[3, i < V - 20] = low
    m[4, V // 2] = np.nan
    m[5, V - 1] = np.inf
    m[6] = low
    m[7, rng.random(V) < 0.5] = -np.inf
    m[8, i >= 3] = low
    return np.concatenate([np.stack(x), m])


def check(lib, rows, V, top, dtype, ld=None, offset=0, seed=0):
    """`rows` rows of the kinds above in turn; every row compared, its values the kind's."""
    import torch
    rng = np.random.default_rng(seed)
    dt = getattr(torch, dtype)
    kinds = torch.from_numpy(rows_of(rng, V, dtype)).to(dt)
    kinds64 = kinds.double().numpy()
    nk = len(kinds64)
    ld = ld or V
    buf = torch.full((offset + rows * ld + 32,), float("nan"), dtype=dt, device="cuda")
    x = buf.as_strided((rows, V), (ld, 1), offset)
    kinds = kinds.cuda()
    for r0 in range(0, rows, nk):
        x[r0:r0 + nk] = kinds[:min(nk, rows - r0)]
    ktargets = rng.integers(0, V, nk)
    ktargets[1], ktargets[3] = -1, V
    t = torch.from_numpy(ktargets.astype(np.int32)).cuda()[torch.arange(rows, device="cuda") % nk]
    r = lib.mca_token_logprobs(x, t, top=top)
    want = R.logprobs(kinds64, ktargets, top)
    which = np.arange(rows) % nk
    for k in ("lse", "entropy", "logprob"):
        got, w, tol = getattr(r, k).double().cpu().numpy(), want[k][which], want["tol_" + k][which]
        fin = np.isfinite(w)
        assert np.array_equal(np.where(fin, 0.0, got), np.where(fin, 0.0, w), equal_nan=True), k
        err = np.abs(got[fin] - w[fin])
        bad = np.flatnonzero(err > tol[fin])
        assert bad.size == 0, (k, which[fin][bad[:5]], err[bad[:5]], tol[fin][bad[:5]])
    if top == 0:
        return
    assert np.array_equal(r.top_index.cpu().numpy(), want["top_index"][which])
    got, w = r.top_logprob.double().cpu().numpy(), want["top_logprob"][which]
    fin = np.isfinite(w)
    assert np.array_equal(np.where(fin, 0.0, got), np.where(fin, 0.0, w), equal_nan=True)
    tol = want["tol_lse"][which][:, None] + 3 * R.U * (np.abs(w) + np.abs(np.where(fin, w, 0)).max())
    assert np.all(np.abs(got[fin] - w[fin]) <= tol[fin])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("top", [0, 8, 32])
@pytest.mark.parametrize("rows,V,pad,offset", [
    # two warps per row
    (1300, 2049, 0, 0), (1300, 9001, 3, 1), (2048, 4099, 0, 0), (1217, 20011, 5, 0),
    # one
    (2500, 3001, 0, 0), (2500, 9001, 7, 3), (4100, 1111, 0, 0), (2433, 33003, 0, 0), (3000, 700, 0, 5),
    (2500, 300, 1, 0),
    # four, eight
    (700, 5003, 1, 1), (200, 40009, 0, 0)])
def test_many_long_rows(gpu_lib, rows, V, pad, offset, top, dtype):
    check(gpu_lib, rows, V, top, dtype, V + pad, offset, seed=V)


@pytest.mark.parametrize("top", [1, 2, 7, 20, 31, 32])
@pytest.mark.parametrize("rows", [5000, 2400, 1000, 9])
def test_any_number_of_alternatives(gpu_lib, rows, top):
    check(gpu_lib, rows, 2333, top, "float32", seed=top)
