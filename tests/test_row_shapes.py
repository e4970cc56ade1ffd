"""The rules that give rows of logits their kernels, compiled for the host: every kernel has sizes in the GPU tests, those that
these tests are written for, and rules change over at the sizes that they name (CPU)."""
import os
import subprocess

import pytest

import test_distill_gpu as D
import test_distill_turns_gpu as T
import test_draw_gpu as S
import test_draw_steps_gpu as SS
from test_answers_gpu import DT

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def n_of(dtype):
    return 4 if dtype == "float32" else 8


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    """f(list of (rows, vocab, dtype, tail)): [(the loss's kernel, n, split), (a draw's warps, split, one round)] of each."""
    exe = str(tmp_path_factory.mktemp("shapes") / "row_shapes_host")
    subprocess.run(["g++", "-std=c++17", "-x", "c++", "-I", os.path.join(ROOT, "paper_2607_08406_gb300", "csrc"), "-o", exe,
                    os.path.join(HERE, "row_shapes_host.cu")], check=True)

    def ask(sizes):
        text = "\n".join(f"{r} {v} {n_of(dt)} {int(tail)}" for r, v, dt, tail in sizes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(sizes)
        got = []
        for line in out:
            by, *v = line.split()
            v = [int(k) for k in v]
            got.append(((by, v[0], v[1]), (v[2], v[3], bool(v[4]))))
        return got
    return ask


def test_rows_in_turn_are_those_of_ctas_that_stay(shapes):
    assert all(d[0] == "staying" for d, _ in shapes(T.STAYING))
    assert all(d[0] == "staying" for d, _ in shapes([(r, v, "bfloat16", False) for r, v in T.CAPTURED]))
    assert shapes([(*T.CAPTURED[1], "bfloat16", True)])[0][0][0] == "staying"
    # of every type, with tail and without, and with two and three rows to a CTA of which some have one less
    assert {(dt, tail) for _, _, dt, tail in T.STAYING} == {(dt, tail) for dt in DT for tail in (False, True)}
    assert {-(-r // 456) for r, *_ in T.STAYING} == {2, 3} and any(r % 456 for r, *_ in T.STAYING)
    assert all(d[:2] == ("team", 4) for d, _ in shapes([(r, v, dt, False) for r, v, dt in T.IN_BETWEEN]))


def test_rows_in_shared_memory_up_to_the_largest(shapes):
    for dtype in DT:
        for last in (False, True):
            for border, more in T.PIECES:
                pieces = T.pieces_of(border, more)
                v = T.vocab_of(pieces, dtype, last)
                assert (v + 2 * n_of(dtype) - 2) // n_of(dtype) == pieces
                with_tail, without = (d[0] for d, _ in shapes([(611, v, dtype, True), (611, v, dtype, False)]))
                assert (with_tail == "shared") == (pieces <= T.MOST) and (without == "shared") == (pieces <= T.LEAST)


def test_every_kernel_of_the_loss_is_tested(shapes):
    sizes = [(r, v, dt, tail) for r, v, _ in D.SIZES for dt in DT for tail in (False, True)]
    sizes += T.STAYING + [(r, v, dt, False) for r, v, dt in T.IN_BETWEEN]
    sizes += [(611, T.vocab_of(T.pieces_of(*b), dt, last), dt, tail) for b in T.PIECES for dt in DT
              for last in (False, True) for tail in (False, True)]
    sizes += [(620, v, dt, tail) for v in (290, 1201, 5003, 12001, 24001) for dt in ("float32", "bfloat16")
              for tail in (False, True)]
    seen = {}
    for size, (d, _) in zip(sizes, shapes(sizes)):
        seen.setdefault(d[:2], []).append(size)
    # every kernel that there is, whatever the size
    grid = [(r, v, dt, tail) for r in (1, 5, 150, 607, 608, 609, 911, 912, 1162, 1163, 1368, 1369, 1551, 3000, 60000)
            for v in (1, 60, 130, 250, 500, 1000, 2000, 4000, 8000, 8191, 8192, 16383, 16384, 26000, 50001, 1 << 20, (1 << 20) + 1)
            for dt in ("float32", "bfloat16") for tail in (False, True)]
    kernels = {d[:2] for d, _ in shapes(grid)}
    assert kernels == {("registers", 1), ("registers", 2), ("registers", 4), ("registers", 8), ("shared", 1),
                       ("shared", 2), ("shared", 4), ("staying", 8), ("team", 4), ("team", 8)}
    assert set(seen) == kernels
    for k in (("staying", 8), ("team", 4), ("team", 8), ("shared", 4)):
        assert {tail for *_, tail in seen[k]} == {False, True}, k


def test_draws_by_one_to_eight_warps_and_clusters(shapes):
    got = [s for _, s in shapes([(r, p * 4, "float32", False) for r, p in SS.SHAPES])]
    assert got == [(1, 1, False), (2, 1, False), (4, 1, False), (8, 1, False), (8, 8, False)]
    assert got == [s for _, s in shapes([(r, p * 8, "bfloat16", False) for r, p in SS.SHAPES])]
    seen = {s for _, s in shapes([(r, v, dt, False) for r, v in S.SIZES for dt in DT])}
    assert any(one for *_, one in seen) and {w for w, *_ in seen} == {1, 2, 4, 8} and {c for _, c, _ in seen} >= {1, 2, 8}
