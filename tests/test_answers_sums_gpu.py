"""How far the sums of log probabilities may be off where a row's values make roundings add up (needs a GPU).

Half steps of fp32 (U = 2^-24 of a value) are counted as the kernel adds: a thread's terms one after the other, then the
threads'. A term exp(d), d = x - m, goes through the difference, its product with log2 e and ex2 (documented: 2
steps, 4 U): 2 |d| + 4 with |d| up to 1 more than from the largest logit. When the reference m is raised by c, the sum is
multiplied by exp(c): 2 |c| + 5, and a part that lies d below goes through at most |d| such raises of 1 or more, and
through one at each join of two threads' sums (the 2 |c| of all of them are within the 9 |d|)."""
import numpy as np
import pytest

import answers_reference as R

pytestmark = pytest.mark.gpu
U = R.U


def logits_of(lib, base, rows, top=0):
    """Row r: base[r % len(base)]."""
    import torch
    b = torch.from_numpy(base.astype(np.float32)).cuda()
    x = b[torch.arange(rows, device="cuda") % len(base)]
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    return lib.mca_token_logprobs(x, t, top=top)


def check(r, base, rows, adds):
    """adds: additions of a thread's longest chain."""
    want = R.logprobs(base, np.zeros(len(base), int), 0)
    adds = adds + 6 * (5 + 3 + 3)                 # joins: the warp's lanes, the row's warps, the cluster's CTAs
    for k, x in enumerate(base):
        d = x - x.max()
        p = np.exp(d) / np.exp(d).sum()
        a = np.abs(d)
        ls, H = np.log(np.exp(d).sum()), want["entropy"][k]
        rel = (p * (9 * a + 13)).sum() + adds                             # of s
        tol = {"lse": rel + 3 * abs(ls) + abs(want["lse"][k]),
               "logprob": rel + 3 * abs(ls) + a[0] + abs(want["logprob"][k])}
        # u: terms as those of s and two roundings more; shifts by up to 1, of which s takes part
        tol["entropy"] = rel + 3 * abs(ls) + (p * a * (9 * a + 17 + adds)).sum() + (p * a).sum() * (rel + 2) + 8 + H
        for name, t in tol.items():
            got = getattr(r, name).double().cpu().numpy()[k::len(base)]
            err = np.abs(got - want[name][k]).max() / U
            assert err <= 1.01 * t, (k, name, err, t)


def chain(V, warps, per_piece=4):
    """fp32 additions of the two halves of a thread's pieces, where each goes to the sums by itself."""
    return per_piece // 2 * -(-(V // per_piece + 2) // (32 * warps)) + 1


# rows that a warp, two, four or eight have
ROWS = [(2433, 1), (1300, 2), (700, 4), (40, 8)]


@pytest.mark.parametrize("rows,warps", ROWS)
@pytest.mark.parametrize("V", [4099, 80011])
def test_rows_that_rise_once(gpu_lib, rows, warps, V):
    """A few symbols 3 to 8 below the others, first: the largest logit is not the first that a thread sees. Its terms
    must not be held at e^8 of what the reference says, nor its entropy be what is left of them."""
    base = []
    for v in (7.9, 7.77, 6.1, 3.3):
        for low in (1024, 40, 1):
            x = np.full(V, v, np.float32).astype(np.float64)
            x[:low] = 0.0
            base.append(x)
    check(logits_of(gpu_lib, np.stack(base), rows), np.stack(base), rows, chain(V, warps))


@pytest.mark.parametrize("rows,warps", ROWS)
def test_one_likely_symbol(gpu_lib, rows, warps):
    """Two symbols that count, 0.4 to 8 apart, the larger behind the other in the same thread's pieces, or elsewhere."""
    V, base = 4099, []
    rng = np.random.default_rng(warps)
    for g in (0.4, 0.9, 1.1, 4.0, 7.5, 7.99, 8.2):
        for gap in (1, 4 * 32 * warps, 1001):
            x = np.full(V, -80.0)
            i = int(rng.integers(0, 1500))
            x[i], x[i + gap] = 0.0, np.float32(g)
            base.append(x)
    check(logits_of(gpu_lib, np.stack(base), rows), np.stack(base), rows, 6)


@pytest.mark.parametrize("rows,warps", ROWS)
@pytest.mark.parametrize("step", [0.002, 0.03, 0.25, 3.0])
def test_rows_that_rise_all_the_way(gpu_lib, rows, warps, step):
    """Each piece larger than the last: a rescaling for each kLead of it at most."""
    V = 8005
    x = (np.arange(V) // 4 * np.float32(step)).astype(np.float32).astype(np.float64)
    base = np.stack([x, x - x.max(), x - 100.0])
    check(logits_of(gpu_lib, base, rows), base, rows, chain(V, warps))


def group_chain(V, warps, per_piece):
    """The same where a thread's pieces come in eight groups, whose sums are added."""
    pieces = -(-(V // per_piece + 2) // (32 * warps))
    return per_piece // 2 * -(-pieces // 8) + 1 + 8 * 6


@pytest.mark.parametrize("rows,warps,V", [(2433, 1, 160003), (2433, 1, 33001), (1300, 2, 120001), (700, 4, 80001)])
def test_long_rows_of_few_values(gpu_lib, rows, warps, V):
    """Few largest logits and a common value below them, whose roundings have one sign: they may add up over a thread's
    group of pieces, not over all of them."""
    base = []
    for v in (-0.2613, -2.3005, -2.3203, -3.6999, -1.226, -0.7):
        x = np.full(V, np.float32(v), np.float32).astype(np.float64)
        x[:132 * warps] = 0.0                     # every thread has one
        base.append(x)
    base.append(np.where(np.arange(V) % 3, 0.0, np.float32(-0.7).astype(np.float64)))
    check(logits_of(gpu_lib, np.stack(base), rows), np.stack(base), rows, group_chain(V, warps, 4))
