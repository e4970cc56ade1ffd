"""Logits and gradient in any two places (needs a GPU): rows between each other's, at different distances from 16-byte
boundaries, with different row distances, above the vocabularies of the small kernels too."""
import numpy as np
import pytest

import answers_reference as R

pytestmark = pytest.mark.gpu
DT = ["float32", "float16", "bfloat16"]


def f64(t):
    return t.double().cpu().numpy()


def inputs(rows, vocab, seed):
    import torch
    rng = np.random.default_rng(seed)
    t = rng.integers(0, vocab, rows)
    t[rows // 2] = -1
    return (3 * rng.standard_normal((rows, vocab)), t, torch.from_numpy(t.astype(np.int32)).cuda(),
            rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32))


def check(lib, logits, out, t, tg, gl, ge, dtype):
    import torch
    x = f64(logits)
    r = lib.mca_token_logprobs(logits, tg)
    lib.mca_token_logprobs_backward(logits, tg, r.lse, r.entropy, torch.from_numpy(gl).cuda(),
                                    torch.from_numpy(ge).cuda(), out=out)
    want, tol = R.backward(x, t, f64(r.lse), f64(r.entropy), gl, ge, dtype)
    assert np.all(np.abs(f64(out) - want) <= tol)
    return x


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,vocab,gap", [(5, 2048, 0), (3, 1031, 0), (9, 10, 6), (4, 4001, 15), (2, 16, 0)])
@pytest.mark.parametrize("first", ["logits", "grad"])
def test_gradient_between_the_rows(gpu_lib, rows, vocab, gap, first, dtype):
    """Two column blocks of one matrix: no element is shared, nothing but the gradient is written."""
    import torch
    x, t, tg, gl, ge = inputs(rows, vocab, vocab)
    wide = torch.full((rows, 2 * vocab + gap), 77.0, dtype=getattr(torch, dtype), device="cuda")
    a, b = wide[:, :vocab], wide[:, vocab + gap:]
    logits, out = (a, b) if first == "logits" else (b, a)
    logits.copy_(torch.from_numpy(x))
    x = check(gpu_lib, logits, out, t, tg, gl, ge, dtype)
    assert np.array_equal(f64(logits), x)
    assert bool((wide[:, vocab:vocab + gap] == 77).all())


def test_shared_elements_are_refused(gpu_lib):
    """One element in common, in the same or a neighbouring row: refused before a launch. Next to it: accepted."""
    import torch
    rows, vocab, ld = 4, 40, 100
    buf = torch.randn(3000, device="cuda")
    v = torch.zeros(rows, device="cuda")
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    logits = buf.as_strided((rows, vocab), (ld, 1), 1000)
    for off, ld2, ok in [(vocab - 1, ld, False), (vocab, ld, True), (1 - vocab, ld, False), (-vocab, ld, True),
                         (ld - vocab, ld, True), (ld - vocab + 1, ld, False), (2 * ld + 3, ld, False),
                         (3 * ld + vocab - 1, ld, False), (3 * ld + vocab, ld, True), (4 * ld, ld, True),
                         (-3 * ld - vocab + 1, ld, False), (-3 * ld - vocab, ld, True), (1, ld, False), (0, ld, True),
                         (0, ld + 1, False), (vocab, ld + 1, False), (3 * ld + vocab, ld + 1, True)]:
        out = buf.as_strided((rows, vocab), (ld2, 1), 1000 + off)
        if ok:
            gpu_lib.mca_token_logprobs_backward(logits, t, v, None, v, out=out)
            continue
        with pytest.raises(gpu_lib.MCAError) as e:
            gpu_lib.mca_token_logprobs_backward(logits, t, v, None, v, out=out)
        assert e.value.status == gpu_lib.MCA_ERR_INVALID


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,vocab,ld,ldg,off,offg", [
    (5, 1025, 1040, 1025, 0, 0), (3, 50001, 50008, 50001, 0, 0), (4, 2048, 2048, 2056, 0, 1), (1, 9001, 9001, 9001, 3, 0),
    (6, 4097, 4097, 4104, 1, 5), (300, 1111, 1120, 1111, 0, 0), (2, 1024, 1030, 1024, 1, 0)])
def test_gradient_of_padded_logits(gpu_lib, rows, vocab, ld, ldg, off, offg, dtype):
    """Logits and gradient at different distances from 16-byte boundaries."""
    import torch
    x, t, tg, gl, ge = inputs(rows, vocab, rows)
    dt = getattr(torch, dtype)
    logits = torch.full((rows * ld + off + 32,), float("nan"), dtype=dt, device="cuda").as_strided((rows, vocab), (ld, 1), off)
    logits.copy_(torch.from_numpy(x))
    buf = torch.full((rows * ldg + offg + 32,), 77.0, dtype=dt, device="cuda")
    out = buf.as_strided((rows, vocab), (ldg, 1), offg)
    check(gpu_lib, logits, out, t, tg, gl, ge, dtype)
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep.as_strided((rows, vocab), (ldg, 1), offg).fill_(False)
    assert bool((buf[keep] == 77).all())
