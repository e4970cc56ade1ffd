"""The answers' entry points refuse bad arguments on the host (CPU only: no kernel runs)."""
import ctypes

import numpy as np
import pytest

from paper_2607_08406_gb300 import build as B
from paper_2607_08406_gb300 import mca


@pytest.fixture(scope="module")
def lib():
    B.build()
    return mca.load_library()


BUF = np.zeros(1 << 12, np.float32)
P = BUF.ctypes.data


def test_struct_layouts_match_header(tmp_path):
    import os
    import subprocess
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                          "mca.h")
    structs = {"mca_code_linear_args": mca.mca_code_linear_args,
               "mca_token_logprobs_args": mca.mca_token_logprobs_args,
               "mca_token_logprobs_backward_args": mca.mca_token_logprobs_backward_args}
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{header}"', "int main(){"]
    for s, cls in structs.items():
        lines.append(f'printf("{s} %zu\\n", sizeof({s}));')
        for f, _ in cls._fields_:
            lines.append(f'printf("{s}.{f} %zu\\n", offsetof({s}, {f}));')
    lines.append("return 0;}")
    c = tmp_path / "probe.c"
    c.write_text("\n".join(lines))
    subprocess.run(["gcc", "-O0", str(c), "-o", str(tmp_path / "probe")], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(tmp_path / "probe")], capture_output=True,
                                                   text=True, check=True).stdout.splitlines())
    for s, cls in structs.items():
        assert int(got[s]) == ctypes.sizeof(cls), s
        for f, _ in cls._fields_:
            assert int(got[f"{s}.{f}"]) == getattr(cls, f).offset, (s, f)


def quantize(lib, x=P, dtype=0, rows=2, cols=8, ldx=8, codes=P, ldc=8, scale=P):
    return lib.mca_quantize_rows(x, dtype, rows, cols, ldx, codes, ldc, scale, None)


def test_quantize_refusals(lib):
    assert quantize(lib, rows=0, x=None) == mca.MCA_OK
    for kw, word in [(dict(dtype=3), b"dtype"), (dict(dtype=-1), b"dtype"), (dict(rows=-1), b"rows"),
                     (dict(rows=1 << 31), b"rows"), (dict(cols=0), b"cols"),
                     (dict(cols=1 << 31, ldx=1 << 31, ldc=1 << 31), b"cols"),
                     (dict(ldx=7), b"x: row"), (dict(ldc=7), b"codes: row"),
                     (dict(ldx=1 << 62), b"row distance"), (dict(x=None), b"x is NULL"),
                     (dict(codes=None), b"codes is NULL"), (dict(scale=None), b"scale is NULL"),
                     (dict(x=P + 2), b"aligned"), (dict(scale=P + 1), b"aligned")]:
        assert quantize(lib, **kw) == mca.MCA_ERR_INVALID, kw
        assert word in lib.mca_last_error(None), (kw, lib.mca_last_error(None))
    # host memory
    assert quantize(lib) == mca.MCA_ERR_INVALID


def linear_args(**kw):
    a = dict(rows=2, n_in=16, n_out=3, x=P, ldx=16, x_scale=P, w=P, ldw=16, w_scale=P, bias=None,
             y=P, ldy=3, dtype=0, act=0, act_param=0.0, workspace=None, workspace_bytes=0,
             stream=None)
    a.update(kw)
    return mca.mca_code_linear_args(**a)


def test_code_linear_refusals(lib):
    n = ctypes.c_size_t(0)
    assert lib.mca_code_linear(ctypes.byref(linear_args(rows=0, x=None))) == mca.MCA_OK
    assert lib.mca_code_linear(None) == mca.MCA_ERR_INVALID
    assert lib.mca_code_linear_workspace_size(ctypes.byref(linear_args()), None) == \
        mca.MCA_ERR_INVALID
    for kw, word in [(dict(rows=-1), b"rows"), (dict(n_in=0), b"n_in"),
                     (dict(n_in=131072, ldx=131072, ldw=131072), b"n_in"), (dict(n_out=0), b"n_out"),
                     (dict(n_out=(1 << 30) + 1, ldy=1 << 31), b"n_out"),
                     (dict(dtype=5), b"dtype"), (dict(act=6), b"transfer"),
                     (dict(act=-1), b"transfer"), (dict(ldx=15), b"x: row"),
                     (dict(ldw=15), b"w: row"), (dict(ldy=2), b"y: row")]:
        a = linear_args(**kw)
        assert lib.mca_code_linear(ctypes.byref(a)) == mca.MCA_ERR_INVALID, kw
        assert word in lib.mca_last_error(None), kw
        assert lib.mca_code_linear_workspace_size(ctypes.byref(a), ctypes.byref(n)) == \
            mca.MCA_ERR_INVALID
    for f in ("x", "x_scale", "w", "w_scale", "y"):
        a = linear_args(**{f: None})
        assert lib.mca_code_linear(ctypes.byref(a)) == mca.MCA_ERR_INVALID
        assert f.encode() + b" is NULL" in lib.mca_last_error(None)
    for f in ("x_scale", "w_scale", "bias", "y"):
        a = linear_args(**{f: P + 2})
        assert lib.mca_code_linear(ctypes.byref(a)) == mca.MCA_ERR_INVALID
        assert b"aligned" in lib.mca_last_error(None)
    assert lib.mca_code_linear(ctypes.byref(linear_args())) == mca.MCA_ERR_INVALID   # host memory
    # operands whose rows do not start on 16-byte boundaries need workspace
    a = linear_args(ldw=17)
    assert lib.mca_code_linear_workspace_size(ctypes.byref(a), ctypes.byref(n)) == mca.MCA_OK
    if n.value:
        assert lib.mca_code_linear(ctypes.byref(a)) == mca.MCA_ERR_OOM
        a.workspace, a.workspace_bytes = P, n.value - 1
        assert lib.mca_code_linear(ctypes.byref(a)) == mca.MCA_ERR_OOM


def logprob_args(**kw):
    a = dict(logits=P, dtype=0, vocab=8, rows=2, ld=8, targets=P, logprob=P, entropy=P, lse=P, top=2,
             top_logprob=P, top_index=P, stream=None)
    a.update(kw)
    return mca.mca_token_logprobs_args(**a)


def test_token_logprobs_refusals(lib):
    assert lib.mca_token_logprobs(None) == mca.MCA_ERR_INVALID
    assert lib.mca_token_logprobs(ctypes.byref(logprob_args(rows=0, logits=None))) == mca.MCA_OK
    for kw, word in [(dict(dtype=9), b"dtype"), (dict(rows=-2), b"rows"), (dict(vocab=0), b"vocab"),
                     (dict(vocab=(1 << 30) + 1, ld=1 << 31), b"vocab"),
                     (dict(ld=7), b"logits: row"), (dict(top=-1), b"top"), (dict(top=33), b"top"),
                     (dict(top=0), b"top = 0"), (dict(targets=None), b"targets"),
                     (dict(logits=None), b"logits is NULL"),
                     (dict(top_logprob=None), b"top_logprob is NULL"),
                     (dict(top_index=None), b"top_index is NULL"), (dict(logits=P + 2), b"aligned"),
                     (dict(targets=P + 2), b"aligned"), (dict(), b"device")]:
        assert lib.mca_token_logprobs(ctypes.byref(logprob_args(**kw))) == mca.MCA_ERR_INVALID, kw
        assert word in lib.mca_last_error(None), (kw, lib.mca_last_error(None))


def backward_args(**kw):
    a = dict(logits=P, dtype=0, vocab=8, rows=2, ld=8, targets=P, lse=P, entropy=P, g_logprob=P,
             g_entropy=P, grad=P, ldg=8, stream=None)
    a.update(kw)
    return mca.mca_token_logprobs_backward_args(**a)


def test_backward_refusals(lib):
    assert lib.mca_token_logprobs_backward(None) == mca.MCA_ERR_INVALID
    assert lib.mca_token_logprobs_backward(ctypes.byref(backward_args(rows=0))) == mca.MCA_OK
    for kw, word in [(dict(dtype=9), b"dtype"), (dict(rows=-2), b"rows"), (dict(vocab=0), b"vocab"),
                     (dict(ld=7), b"logits: row"), (dict(ldg=7), b"grad: row"),
                     (dict(g_logprob=None, g_entropy=None), b"neither"),
                     (dict(targets=None), b"targets"), (dict(entropy=None), b"entropy"),
                     (dict(lse=None), b"lse is NULL"), (dict(grad=None), b"grad is NULL"),
                     (dict(lse=P + 1), b"aligned")]:
        assert lib.mca_token_logprobs_backward(ctypes.byref(backward_args(**kw))) == \
            mca.MCA_ERR_INVALID, kw
        assert word in lib.mca_last_error(None), (kw, lib.mca_last_error(None))


def test_handle_calls_refuse_null(lib):
    n = ctypes.c_size_t(0)
    assert lib.mca_score(None, P, 0, P, P, P, None, None) == mca.MCA_ERR_INVALID
    assert lib.mca_predict(None, P, 1, 8, P, None, 0) == mca.MCA_ERR_INVALID
    assert lib.mca_predict_workspace_size(None, 1, ctypes.byref(n)) == mca.MCA_ERR_INVALID


def test_binding_refuses_wrong_tensors():
    """The binding's own checks come before any device work."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 8)
    for call in (lambda: mca.mca_quantize_rows(x), lambda: mca.mca_token_logprobs(x),
                 lambda: mca.mca_code_linear(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0]),
                 lambda: mca.mca_token_logprobs_backward(x, None, x[:, 0], None, None)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        mca._dtype_code(torch.float64)
