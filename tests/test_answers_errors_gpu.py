"""An error that one call has returned is not returned again by the next (needs a GPU)."""
import numpy as np
import pytest

import answers_reference as R
from paper_2607_08406_gb300 import workloads as W

pytestmark = pytest.mark.gpu


def out_of_memory(gpu_lib):
    """A handle whose own workspace is larger than any device's memory: refused by the allocation itself."""
    import torch
    N, H = 100_000_000, 16384                              # fields of 6.5 TB
    layers = [W.Layer(1, H, "tanh", 0.0, "fp32", 1.0), W.Layer(H, 10, "identity", 0.0, "fp32", 1.0)]
    with pytest.raises(gpu_lib.MCAError) as e:
        gpu_lib.mca_create(layers, "softmax_ce", W.Domain(), torch.zeros(N, 1, device="cuda"),
                           torch.zeros(N, dtype=torch.int32, device="cuda"), np.zeros(11 * H, np.float32),
                           torch_workspace=False)
    assert e.value.status == gpu_lib.MCA_ERR_OOM


def small_net():
    rng = np.random.default_rng(0)
    layers = [W.Layer(20, 8, "tanh", 0.0, "fp32", 1.0), W.Layer(8, 4, "identity", 0.0, "fp32", 1.0)]
    return W.MLPWorkload("errors", layers, "softmax_ce", W.synth_images(rng, 50, 20, 0.3),
                         rng.integers(0, 4, 50).astype(np.int32), W.uniform_init(rng, layers, 0.2), 20, 8)


@pytest.mark.parametrize("what", ["score", "quantize", "linear", "grad", "handle", "create"])
def test_calls_after_an_allocation_that_failed(gpu_lib, what):
    import torch
    h = gpu_lib.create_from_workload(small_net())
    x = torch.randn(4, 300, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    r = gpu_lib.mca_token_logprobs(x, t)
    i8, one = torch.ones(4, 32, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    out_of_memory(gpu_lib)
    if what == "score":
        want = R.logprobs(x.double().cpu().numpy(), np.zeros(4, int), 0)
        got = gpu_lib.mca_token_logprobs(x, t).lse.double().cpu().numpy()
        assert np.all(np.abs(got - want["lse"]) <= want["tol_lse"])
    elif what == "quantize":
        q, s = gpu_lib.mca_quantize_rows(x)
        assert np.array_equal(q.cpu().numpy(), R.quantize(x.double().cpu().numpy())[0])
    elif what == "linear":
        y = torch.zeros(4, 4, device="cuda")
        gpu_lib.mca_code_linear(i8, one, i8, one, out=y, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
        assert bool((y == 32).all())
    elif what == "grad":
        g = gpu_lib.mca_token_logprobs_backward(x, t, r.lse, None, one)
        assert abs(float(g.sum())) <= 1e-4
    elif what == "handle":
        logits, s = gpu_lib.mca_score(h, 1)
        assert gpu_lib.mca_predict(h, torch.randn(3, 20, device="cuda")).shape == (3, 4)
        assert np.isfinite(gpu_lib.mca_loss(h))               # and the handle stays usable
    else:
        assert np.isfinite(gpu_lib.mca_loss(gpu_lib.create_from_workload(small_net())))
