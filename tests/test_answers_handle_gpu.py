"""mca_score and mca_predict: a handle's answers on its own samples and on new ones (needs a GPU)."""
import numpy as np
import pytest

import answers_reference as R
from oracle import mca_oracle as O
from oracle import mca_tfm as T
from paper_2607_08406_gb300 import workloads as W

pytestmark = pytest.mark.gpu


def net(rng, dims, hidden, out, loss, N, wkind="fp32", gamma=1.0):
    scale = [2.0 ** -4, 2.0 ** -6] if wkind == "ternary_i8" else [1.0] * (len(dims) - 1)
    layers = [W.Layer(dims[m], dims[m + 1], hidden if m + 2 < len(dims) else out,
                      gamma if hidden == "gaussian" and m + 2 < len(dims) else 0.0, wkind, scale[m])
              for m in range(len(dims) - 1)]
    init = W.uniform_init(rng, layers, 0.2)
    if wkind == "ternary_i8":
        init = rng.integers(-1, 2, len(init)).astype(np.float32)
    return W.MLPWorkload("answers", layers, loss, W.synth_images(rng, N, dims[0], 0.3),
                         rng.integers(0, dims[-1], N).astype(np.int32), init, 200, 16)


def check_score(gpu_lib, h, logits, targets, top, atol):
    """mca_score's logits within atol of `logits` (fp64), and its answers those of its own logits."""
    got, r = gpu_lib.mca_score(h, top)
    z = got.double().cpu().numpy()
    assert np.abs(z - logits).max() <= atol
    want = R.logprobs(z, targets, top)
    for k in ("logprob", "entropy", "lse"):
        assert np.all(np.abs(getattr(r, k).double().cpu().numpy() - want[k]) <= want["tol_" + k]), k
    if top:
        assert np.array_equal(r.top_index.cpu().numpy(), want["top_index"])
    L = -float(r.logprob.double().sum()) / len(targets)
    assert abs(L - gpu_lib.mca_loss(h)) <= 1e-5 * abs(L)


@pytest.mark.parametrize("dims,act,N,top", [((40, 33, 10), "tanh", 1003, 1), ((20, 8, 2), "relu", 77, 5),
                                            ((30, 16, 16, 7), "gelu", 300, 3),
                                            ((50, 256, 256, 256, 10), "tanh", 700, 0)])
def test_score_mlp(gpu_lib, dims, act, N, top):
    rng = np.random.default_rng(N)
    wl = net(rng, dims, act, "identity", "softmax_ce", N)
    h = gpu_lib.create_from_workload(wl)
    for _ in range(2):                       # at the start, and after a run has moved the state
        p = O.Params(wl.layers, gpu_lib.mca_get_params(h, wl.n_params))
        a = O.forward(p, wl.X.T.astype(np.float64))[1].T
        # fp32 fields of up to 256 terms per layer, kept up incrementally
        check_score(gpu_lib, h, a, wl.y, top, 1e-4 * max(1.0, np.abs(a).max()))
        gpu_lib.mca_run(h, 200, 5)


@pytest.mark.parametrize("vocab,ctx,d,layers,heads,ff,B,act", [
    (65, 64, 128, 2, 4, 256, 6, "gelu"), (50, 21, 24, 1, 2, 40, 5, "gaussian")])
def test_score_transformer(gpu_lib, vocab, ctx, d, layers, heads, ff, B, act):
    spec = W.TfmSpec(vocab=vocab, ctx=ctx, d_model=d, n_layer=layers, n_head=heads, d_ff=ff, act=act,
                     act_param=1.0 if act == "gaussian" else 0.0)
    wl = W.char_transformer(batch=B, text_len=3000, spec=spec, n_trials=60, K=8)
    h = gpu_lib.create_from_tfm_workload(wl)
    for _ in range(2):
        flat = gpu_lib.mca_get_params(h, len(wl.init))
        z = T.tfm_forward(spec, flat.astype(np.float64), wl.tokens[:, :ctx]).reshape(-1, vocab)
        check_score(gpu_lib, h, z, wl.tokens[:, 1:].reshape(-1), 5, 2e-4 * max(1.0, np.abs(z).max()))
        gpu_lib.mca_run(h, 60, 3)


def test_score_refuses_mse(gpu_lib):
    wl = net(np.random.default_rng(1), (20, 8, 4), "tanh", "sigmoid", "mse_onehot", 50)
    h = gpu_lib.create_from_workload(wl)
    with pytest.raises(gpu_lib.MCAError) as e:
        gpu_lib.mca_score(h)
    assert e.value.status == gpu_lib.MCA_ERR_UNSUPPORTED
    gpu_lib.mca_run(h, 10, 1)                # the handle stays usable


def layer_by_layer(gpu_lib, wl, params, codes, x):
    """The chain that mca_predict documents, from the operators."""
    import torch
    at, cur = 0, x
    for m, L in enumerate(wl.layers):
        n = L.n_in * L.n_out
        if L.wkind == "ternary_i8":
            wq = torch.from_numpy(codes[at:at + n].reshape(L.n_out, L.n_in)).cuda()
            ws = torch.full((L.n_out,), L.scale, device="cuda")
        else:
            wq, ws = gpu_lib.mca_quantize_rows(
                torch.from_numpy(params[at:at + n].reshape(L.n_out, L.n_in)).cuda())
        at += n
        q, s = gpu_lib.mca_quantize_rows(cur)
        half = m + 1 < len(wl.layers) and L.act in ("tanh", "sigmoid", "gaussian")
        cur = gpu_lib.mca_code_linear(q, s, wq, ws, act=L.act, act_param=L.act_param,
                                      dtype=torch.float16 if half else torch.float32)
    return cur


@pytest.mark.parametrize("dims,hidden,out,loss,wkind,n", [
    ((784, 300, 10), "gaussian", "sigmoid", "mse_onehot", "ternary_i8", 500),
    ((39, 50, 7), "gaussian", "sigmoid", "mse_onehot", "masked_fp32", 33),
    ((100, 64, 10), "tanh", "identity", "softmax_ce", "fp32", 1),
    ((100, 100, 100, 10), "relu", "identity", "softmax_ce", "fp32", 129),
    ((64, 256, 256, 256, 10), "tanh", "identity", "softmax_ce", "fp32", 2000)])
def test_predict(gpu_lib, dims, hidden, out, loss, wkind, n):
    """New samples: the operators' chain bit for bit, and near the net's own outputs, with weights that a run
    has changed."""
    import torch
    rng = np.random.default_rng(n)
    wl = net(rng, dims, hidden, out, loss, 200, wkind)
    h = gpu_lib.create_from_workload(wl)
    gpu_lib.mca_run(h, 200, 3)
    params, codes = gpu_lib.mca_get_params(h, wl.n_params), gpu_lib.mca_get_codes(h, wl.n_params)
    S0 = gpu_lib.mca_loss(h)
    wide = torch.randn(n, dims[0] + 3, device="cuda")
    x = wide[:, 1:dims[0] + 1]
    got = gpu_lib.mca_predict(h, x)
    assert torch.equal(got, layer_by_layer(gpu_lib, wl, params, codes, x))
    assert gpu_lib.mca_loss(h) == S0
    # in 64 bits with the effective weights: 8-bit steps are 1/254 of a row's largest value, and the errors of
    # single inputs and weights are independent and uniform: 5 % of the outputs' spread is far outside
    cur, at = x.double().cpu().numpy(), 0
    for L in wl.layers:
        w = params[at:at + L.n_in * L.n_out].astype(np.float64).reshape(L.n_out, L.n_in)
        at += L.n_in * L.n_out
        cur, _ = R.act(L.act, cur @ w.T, L.act_param)
    err = got.double().cpu().numpy() - cur
    assert np.sqrt((err ** 2).mean()) <= 0.05 * max(np.sqrt((cur ** 2).mean()), 1e-3)
    # and scored as the net's answers
    if loss == "softmax_ce":
        t = torch.zeros(n, dtype=torch.int32, device="cuda")
        r = gpu_lib.mca_token_logprobs(got, t, top=1)
        assert torch.equal(r.top_index[:, 0].long(), got.argmax(dim=1))


def test_predict_in_passes(gpu_lib):
    """More samples than go through the layers at once, on a stream of the handle's own."""
    import torch
    rng = np.random.default_rng(2)
    wl = net(rng, (24, 4096, 3), "tanh", "identity", "softmax_ce", 64)
    st = torch.cuda.Stream()
    h = gpu_lib.create_from_workload(wl, stream=st.cuda_stream)
    x = torch.randn(20001, 24, device="cuda")
    for n in (20001, 16384, 8200):
        got = gpu_lib.mca_predict(h, x[:n])
        ref = layer_by_layer(gpu_lib, wl, gpu_lib.mca_get_params(h, wl.n_params), None, x[:n])
        assert torch.equal(got, ref)
    logits, r = gpu_lib.mca_score(h, 2)
    assert logits.shape == (64, 3) and r.top_index.shape == (64, 2)
    assert abs(-float(r.logprob.double().mean()) - gpu_lib.mca_loss(h)) <= 1e-5
    assert gpu_lib.mca_predict(h, x[:0]).shape == (0, 3)


def test_predict_refusals(gpu_lib):
    import ctypes
    import torch
    wl = net(np.random.default_rng(1), (20, 8, 4), "tanh", "identity", "softmax_ce", 50)
    h = gpu_lib.create_from_workload(wl)
    lib = gpu_lib.load_library()
    x = torch.randn(6, 20, device="cuda")
    with pytest.raises(ValueError):
        gpu_lib.mca_predict(h, x[:, :19])
    with pytest.raises(ValueError):
        gpu_lib.mca_predict(h, x.half())
    out = torch.zeros(6, 4, device="cuda")
    need = gpu_lib.mca_predict_workspace_size(h, 6)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    inv, oom = gpu_lib.MCA_ERR_INVALID, gpu_lib.MCA_ERR_OOM
    a = (h.ptr, x.data_ptr(), 6, 20, out.data_ptr(), ws.data_ptr(), need)
    for pos, val, want in [(1, None, inv), (2, -1, inv), (3, 19, inv), (4, None, inv), (5, None, oom),
                           (6, need - 1, oom), (5, ws.data_ptr() + 16, inv)]:
        b = list(a)
        b[pos] = val
        assert lib.mca_predict(*b) == want, pos
    assert lib.mca_predict(*a) == gpu_lib.MCA_OK
    n = ctypes.c_size_t(0)
    tw = W.char_transformer(batch=2, text_len=200, n_trials=5, K=4, spec=W.TfmSpec(
        vocab=20, ctx=8, d_model=16, n_layer=1, n_head=2, d_ff=32))
    ht = gpu_lib.create_from_tfm_workload(tw)
    assert lib.mca_predict_workspace_size(ht.ptr, 3, ctypes.byref(n)) == gpu_lib.MCA_ERR_UNSUPPORTED


def test_predict_refuses_inputs_beyond_exact_sums(gpu_lib):
    """More inputs than an integer sum of 8-bit codes has room for: trained, but not answered in 8 bits."""
    import torch
    for dims in [(131072, 4, 3), (5, 131072, 3)]:
        wl = net(np.random.default_rng(2), dims, "tanh", "identity", "softmax_ce", 20)
        h = gpu_lib.create_from_workload(wl)
        x = torch.ones(2, dims[0], device="cuda")
        for call in (lambda: gpu_lib.mca_predict(h, x), lambda: gpu_lib.mca_predict_workspace_size(h, 2)):
            with pytest.raises(gpu_lib.MCAError, match="131071"):
                call()
        assert np.isfinite(gpu_lib.mca_loss(h))
