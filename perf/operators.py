"""The operators that a trained net's answers are made with, as calls of real size: what is measured.

* "linear"  a layer in 8-bit integers: the inputs' rows are quantised with a scale each, multiplied with
            weights that are kept as codes with a scale per output neuron, and the sums go through scale,
            bias and transfer function
* "score"   log probabilities of given symbols from logits, with each row's entropy and the most probable
            alternatives
* "grad"    the gradient of log probability and entropy with respect to the logits

`run` computes a pass in elementary torch operations, or with the library's entry points where `own` is
true. Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _linear(rows, n_in, n_out, dtype="bf16", act="identity", gamma=0.0, bias=False, ternary=False):
    """dtype: of the inputs and the outputs."""
    return {"op": "linear", "rows": rows, "n_in": n_in, "n_out": n_out, "dtype": dtype, "act": act,
            "gamma": gamma, "bias": bias, "ternary": ternary}


def _score(rows, vocab, dtype="bf16", top=0, masked=0.0):
    """masked: share of the symbols whose logits are -inf."""
    return {"op": "score", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top,
            "masked": masked}


def _grad(rows, vocab, dtype="bf16", masked=0.0, entropy=True):
    return {"op": "grad", "rows": rows, "vocab": vocab, "dtype": dtype, "masked": masked,
            "entropy": entropy}


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # one feed-forward layer of the character-level Transformer on one sequence: latency
    add("linear_chars", _linear(64, 128, 512, "fp32", "gelu", bias=True))
    # a single token through a wide layer: the weights are read once
    add("linear_token", _linear(1, 4096, 16384, "bf16"))
    # a few dozen requests answered together
    add("linear_batch", _linear(48, 4096, 4096, "fp16", bias=True))
    # a hidden layer of odd sizes (the pruned net's), a test set's samples
    add("linear_ragged", _linear(2347, 391, 1001, "fp32", "gaussian", 1.0))
    # the ternary net's hidden layer on all its samples
    add("linear_ternary", _linear(60000, 784, 4096, "fp16", "gaussian", 1.0, ternary=True))
    # a large layer on a long prompt: arithmetic
    add("linear_large", _linear(8192, 8192, 8192, "bf16"))
    # ten classes, every sample of the benchmark's training set, the predicted label
    add("score_classes", _score(60000, 10, "fp32", top=1))
    # next-symbol log probabilities of all windows of the character-level Transformer
    add("score_chars", _score(16384, 65, "fp32", top=5))
    # what is reported beside one sampled token over a large vocabulary
    add("score_token", _score(1, 128000, "bf16", top=20))
    # a text's log probabilities over a vocabulary of odd size, part of it not allowed
    add("score_text", _score(2048, 50001, "bf16", top=8, masked=0.1))
    # the gradient of the same: characters, and the large vocabulary
    add("grad_chars", _grad(16384, 65, "fp32"))
    add("grad_text", _grad(2048, 50001, "bf16", masked=0.1))
    return out


MOST_MACS = 8192.0 ** 3            # of a drawn layer
MOST_LOGITS = 2048 * 50001         # of a drawn scoring call


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rounded(rng, v, to):
    return max(to, v // to * to) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "score", "score", "grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "linear":
        rows = _log_int(rng, 1, 60000)
        n_in = _rounded(rng, _log_int(rng, 64, 16384), 64)
        n_out = _rounded(rng, _log_int(rng, 10, 16384), 64)
        while float(rows) * n_in * n_out > MOST_MACS or rows * max(n_in, n_out) > 60000 * 4096:
            rows = max(1, rows // 2)
        act, gamma = rng.choice([("identity", 0.0), ("identity", 0.0), ("tanh", 0.0),
                                 ("relu", 0.0), ("gelu", 0.0), ("gaussian", 1.0)])
        return _linear(rows, n_in, n_out, dtype, act, gamma, rng.random() < 0.5,
                       rng.random() < 0.25)
    vocab = _log_int(rng, 2, 160000)
    rows = min(_log_int(rng, 1, 60000), max(1, MOST_LOGITS // vocab))
    masked = rng.choice([0.0, 0.0, 0.1, 0.5]) if vocab >= 64 else 0.0
    if op == "score":
        return _score(rows, vocab, dtype, min(vocab, rng.choice([0, 1, 5, 8, 20, 32])), masked)
    return _grad(rows, vocab, dtype, masked, rng.random() < 0.7)


# ------------------------------------------------------------------------------------ inputs

def _plain_codes(x):
    """Codes (as fp32 integers) and scales of x's rows: scale = max |x| / 127 in 32 bits, the quotients
    in 64 bits, so that none is rounded across a half."""
    scale = (x.float().abs().amax(dim=1) / 127.0).float()
    q = torch.round(x.double() / scale.double().clamp_min(1e-300)[:, None])
    q = torch.where(scale[:, None] > 0, q, torch.zeros_like(q)).clamp(-127, 127)
    return q.float(), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    rows = case["rows"]
    st = {"case": case}
    if case["op"] == "linear":
        n_in, n_out = case["n_in"], case["n_out"]
        # inputs of different magnitude from row to row, as activations have
        x = torch.randn(rows, n_in, generator=g, device="cuda")
        x *= torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
        st["x"] = x.to(dt)
        if case["ternary"]:
            st["w"] = torch.randint(-1, 2, (n_out, n_in), generator=g, device="cuda",
                                    dtype=torch.int32).to(torch.int8)
            st["w_scale"] = torch.full((n_out,), 2.0 ** -4, device="cuda")
        else:
            w = torch.randn(n_out, n_in, generator=g, device="cuda") / math.sqrt(n_in)
            q, st["w_scale"] = _plain_codes(w)
            st["w"] = q.to(torch.int8)
            del w, q
        st["bias"] = (0.1 * torch.randn(n_out, generator=g, device="cuda") if case["bias"]
                      else None)
        return st
    vocab = case["vocab"]
    x = 2.0 * torch.randn(rows, vocab, generator=g, device="cuda")
    if case["masked"]:
        off = torch.rand(vocab, generator=g, device="cuda") < case["masked"]
        off[0] = False
        x[:, off] = float("-inf")
    st["logits"] = x.to(dt)
    del x
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    if case["masked"]:
        targets = torch.where(off[targets.long()], torch.zeros_like(targets), targets)
    if rows > 16:                  # padding behind the last sequence
        targets[-(rows // 16):] = -1
    st["targets"] = targets
    if case["op"] == "grad":
        xl = st["logits"].double()
        lse = torch.logsumexp(xl, dim=1)
        lp = xl - lse[:, None]
        p = torch.exp(lp)
        ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(dim=1)
        st["lse"], st["entropy"] = lse.float(), ent.float()
        del xl, lp, p
        st["g_logprob"] = torch.randn(rows, generator=g, device="cuda")
        st["g_entropy"] = (0.1 * torch.randn(rows, generator=g, device="cuda") if case["entropy"]
                           else None)
    return st


# ------------------------------------------------------------------------------------ one pass

def _act(z, act, gamma):
    if act == "tanh":
        return torch.tanh(z)
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    if act == "relu":
        return torch.clamp_min(z, 0.0)
    if act == "gaussian":
        return torch.exp(-gamma * z * z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _plain_linear(st):
    case = st["case"]
    q, scale = _plain_codes(st["x"])
    z = (q @ st["w"].float().t()) * scale[:, None] * st["w_scale"]
    if st["bias"] is not None:
        z = z + st["bias"]
    return [scale, _act(z, case["act"], case["gamma"]).to(st["x"].dtype)]


def _plain_score(st):
    case = st["case"]
    x = st["logits"].float()
    m = x.amax(dim=1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    s = e.sum(dim=1)
    lse = m[:, 0] + torch.log(s)
    t = st["targets"].long()
    at = torch.gather(d, 1, t.clamp_min(0)[:, None])[:, 0]
    logprob = torch.where(t >= 0, at - torch.log(s), torch.zeros_like(s))
    d = torch.where(e > 0, d, torch.zeros_like(d))
    entropy = torch.log(s) - (e * d).sum(dim=1) / s
    out = [logprob, entropy, lse]
    if case["top"]:
        rest = x.clone()
        vals, idx = [], []
        for _ in range(case["top"]):
            i = torch.argmax(rest, dim=1, keepdim=True)      # the first of equal ones
            v = torch.gather(rest, 1, i)
            rest.scatter_(1, i, float("-inf"))
            vals.append(v)
            idx.append(torch.where(v > float("-inf"), i, torch.full_like(i, -1)))
        vals = torch.cat(vals, dim=1)
        out += [(vals - m) - torch.log(s)[:, None], torch.cat(idx, dim=1).int()]
    return out


def _plain_grad(st):
    x = st["logits"].float()
    lp = x - st["lse"][:, None]
    p = torch.exp(lp)
    t = st["targets"].long()
    g = torch.where(t >= 0, st["g_logprob"], torch.zeros_like(st["g_logprob"]))
    dx = -g[:, None] * p
    if st["g_entropy"] is not None:
        lp = torch.where(p > 0, lp, torch.zeros_like(lp))
        dx = dx - (st["g_entropy"][:, None] * p) * (lp + st["entropy"][:, None])
    dx.scatter_add_(1, t.clamp_min(0)[:, None], g[:, None])
    return [dx.to(st["logits"].dtype)]


def _own(st):
    from paper_2607_08406_gb300 import mca
    case = st["case"]
    if case["op"] == "linear":
        q, scale = mca.mca_quantize_rows(st["x"])
        y = mca.mca_code_linear(q, scale, st["w"], st["w_scale"], bias=st["bias"],
                                act=case["act"], act_param=case["gamma"], dtype=st["x"].dtype)
        return [scale, y]
    if case["op"] == "score":
        r = mca.mca_token_logprobs(st["logits"], st["targets"], top=case["top"])
        out = [r.logprob, r.entropy, r.lse]
        return out + [r.top_logprob, r.top_index] if case["top"] else out
    return [mca.mca_token_logprobs_backward(st["logits"], st["targets"], st["lse"], st["entropy"],
                                            st["g_logprob"], st["g_entropy"])]


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "score": _plain_score,
            "grad": _plain_grad}[state["case"]["op"]](state)


def work(case):
    rows, es = case["rows"], BYTES[case["dtype"]]
    if case["op"] == "linear":
        n_in, n_out = case["n_in"], case["n_out"]
        b = rows * n_in * es + n_in * n_out + rows * n_out * es + 4 * (rows + n_out)
        return {"bytes": b + (4 * n_out if case["bias"] else 0),
                "flops": 2.0 * rows * n_in * n_out}
    n = rows * case["vocab"]
    if case["op"] == "score":
        return {"bytes": n * es + rows * (16 + 8 * case["top"]), "flops": 5.0 * n}
    return {"bytes": 2 * n * es + rows * (20 if case["entropy"] else 12), "flops": 6.0 * n}


# ------------------------------------------------------------------------------------ by definition

def exact(case, seed):
    """The definitions in 64 bits, block of rows by block of rows."""
    st = prepare(case, seed)
    rows = case["rows"]
    parts = []
    if case["op"] == "linear":
        w = st["w"].double() * st["w_scale"].double()[:, None]
        step = max(1, (1 << 27) // max(case["n_in"], case["n_out"]))
        for r0 in range(0, rows, step):
            x = st["x"][r0:r0 + step].double()
            s = (x.abs().max(dim=1, keepdim=True).values / 127.0).float().double()
            q = torch.where(s > 0, x / torch.where(s > 0, s, torch.ones_like(s)),
                            torch.zeros_like(x)).round().clamp(-127.0, 127.0)
            z = torch.matmul(q * s, w.t())
            if st["bias"] is not None:
                z += st["bias"].double()
            if case["act"] == "gelu":
                z = z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
            elif case["act"] == "gaussian":
                z = torch.exp(-case["gamma"] * z.square())
            elif case["act"] == "tanh":
                z = torch.tanh(z)
            elif case["act"] == "relu":
                z = torch.maximum(z, torch.zeros_like(z))
            parts.append((s[:, 0], z))
        return [torch.cat(c) for c in zip(*parts)]
    step = max(1, (1 << 25) // case["vocab"])
    for r0 in range(0, rows, step):
        x = st["logits"][r0:r0 + step].double()
        t = st["targets"][r0:r0 + step].long()
        has = t >= 0
        if case["op"] == "score":
            lsm = torch.log_softmax(x, dim=1)
            p = lsm.exp()
            lp = torch.where(has, lsm.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
            part = [lp, -torch.xlogy(p, p).sum(dim=1), torch.logsumexp(x, dim=1)]
            if case["top"]:
                v, i = torch.sort(x, dim=1, descending=True, stable=True)
                v, i = v[:, :case["top"]], i[:, :case["top"]]
                none = torch.isinf(v)
                part += [torch.where(none, v, lsm.gather(1, i)),
                         torch.where(none, -1, i).int()]
        else:
            lp = x - st["lse"][r0:r0 + step].double()[:, None]
            p = lp.exp()
            gl = (st["g_logprob"][r0:r0 + step].double() * has)[:, None]
            hot = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], 1.0)
            dx = gl * (hot - p)
            if st["g_entropy"] is not None:
                ge = st["g_entropy"][r0:r0 + step].double()[:, None]
                dx -= ge * (torch.xlogy(p, p) + p * st["entropy"][r0:r0 + step].double()[:, None])
            part = [dx]
        parts.append(part)
    return [torch.cat(c) for c in zip(*parts)]
