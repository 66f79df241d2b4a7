"""What the host launches for calls of include/topoep_ffn.h, seen without a GPU
(tests/launches.py)."""
import ast
import os
import re

import pytest

import launches
from ffncases import DENSE_FEW, DENSE_LARGE, INT8_FEW, INT8_GROUPS, INT8_LARGE, ROUTED_FEW, ROUTED_LARGE
from launches import BF16, F16, F32


def few_grids(answers):
    return [grid[0] * (4 if name.endswith("1>") else 1) for _, got in answers for name, grid, _ in got
            if name.startswith("few_")]


@pytest.mark.parametrize("T,H,I,E,L,k", [(512, 4096, 4096, 256, 1, 8), (512, 7168, 2048, 256, 8, 8),
                                         (448, 2048, 768, 256, 32, 8), (256, 512, 256, 256, 4, 8)])
def test_few_rows_of_a_share_have_a_grid_of_the_rows_expected(T, H, I, E, L, k, tmp_path):
    """Tiles of 16 rows of weights (8 units of both halves) for spans of 4 rows at least: of twice the expected
    rows and one more a group, or 4096."""
    answers, _ = launches.record([launches.forward(T, H, I, BF16, L, k, E)], tmp_path)
    spans = 2 * -(-T * k * L // E) / 4 + min(L, T * k) + 1
    up, down = few_grids(answers)
    assert up <= max(4100, spans * I / 8) and down <= max(4100, spans * H / 16 + 4)


def test_few_rows_of_experts_that_are_all_here_have_a_tile_each(tmp_path):
    T, H, I, E, k = 64, 2048, 768, 128, 8
    answers, _ = launches.record([launches.forward(T, H, I, BF16, E, k, E)], tmp_path)
    up, down = few_grids(answers)
    # eight columns a tile at most: 512 rows and a remainder of every expert
    assert up >= (512 // 8 + 128) * I // 8 and down >= (512 // 8 + 128) * H // 16


def block_calls(T, H, I, dtype, E=1, L=1, k=0):
    return [launches.forward(T, H, I, dtype, L, k, E, save) for save in (True, False)] + [
        launches.backward(T, H, I, dtype, L, k, E)]


def launched(calls, tmp):
    """The kernels of every call, and all that the three sources have."""
    answers, kernels = launches.record(calls, tmp)
    assert all(rc == 0 for rc, _ in answers)
    for _, got in answers:
        for name, grid, block in got:
            assert all(0 < g * b < 1 << 32 for g, b in zip(grid, block)), (name, grid, block)
    ours = re.compile(r"(up|out|hidden|grad|combine|weights|parts|few_up|few_down|rank|sum|place|quantize|quantize_any|int8|"
                      r"few_int8)_kernel\b")
    return [{name for name, _, _ in got} for _, got in answers], {n for n in kernels if ours.match(n)}


def lists(module, names):
    """Lists of cases of a GPU test, which does not import without a GPU."""
    tree = ast.parse(open(os.path.join(os.path.dirname(__file__), module)).read())
    known = dict(F32=F32, BF16=BF16, F16=F16)
    return [eval(compile(ast.Expression(n.value), module, "eval"), known) for name in names for n in tree.body
            if isinstance(n, ast.Assign) and getattr(n.targets[0], "id", None) == name]


def test_large_and_few_cases_reach_what_they_are_for(tmp_path):
    calls = [c for case in DENSE_LARGE for c in block_calls(*case, BF16)]
    calls += [c for T, H, I, E, L, k in ROUTED_LARGE for c in block_calls(T, H, I, BF16, E, L, k)]
    got, _ = launched(calls, tmp_path)
    got = [got[i] | got[i + 1] | got[i + 2] for i in range(0, len(got), 3)]
    for i, cases in enumerate((got[:5], got[5:])):
        up, hidden, out, of_down, of_up = ({n.replace("Shape<Bf16, 256, 256, 2, 4, ", "<") for n in case} for case in cases)
        routed = ("false", "true")[i]
        assert {"up_kernel<<false, false, 2>, true>", "up_kernel<<false, false, 2>, false>"} <= up
        assert "hidden_kernel<<true, false, 2> >" in hidden
        assert {"out_kernel<<false, false, 2>, false>", "out_kernel<<true, false, 2>, true>"} <= out
        assert "grad_kernel<<true, true, 1>, true, %s>" % routed in of_down
        assert "grad_kernel<<true, true, 1>, false, %s>" % routed in of_up


def test_every_kernel_is_run_by_a_case_of_the_gpu_tests(tmp_path):
    dense, routed = lists("test_gpu_ffn.py", ["DENSE", "ROUTED"])
    shapes, groups = lists("test_gpu_int8.py", ["SHAPES", "GROUPS"])
    calls = [c for T, H, I, dtype in dense for c in block_calls(T, H, I, dtype)]
    calls += [c for T, H, I, E, L, k, dtype in routed for c in block_calls(T, H, I, dtype, E, L, k)]
    for dtype in (BF16, F16):
        calls += [c for T, H, I in DENSE_LARGE + DENSE_FEW for c in block_calls(T, H, I, dtype)]
        calls += [c for T, H, I, E, L, k in ROUTED_LARGE + ROUTED_FEW for c in block_calls(T, H, I, dtype, E, L, k)]
    calls.append(launches.backward(50, 64, 48, BF16, 8, 2, 8, ["weights"]))
    calls += [launches.int8(M, N + N % 2, K, BF16, 0, gated) for M, N, K in shapes for gated in (False, True)]
    calls += [launches.int8(ends[-1], N, K, BF16, len(ends) - 1, gated) for ends, N, K in groups for gated in (False, True)]
    calls += [launches.int8(M, N, K, BF16, 0, gated) for M, N, K, gated in INT8_LARGE + INT8_FEW]
    calls += [launches.int8(ends[-1], N, K, BF16, len(ends) - 1, gated) for ends, N, K, gated in INT8_GROUPS]
    # (the sizes of test_gpu_int8.py's test_quantize and of test_gpu_expert_rows.py)
    calls += [launches.quantize(M, K, dtype) for dtype in (F32, BF16, F16)
              for M, K in ((3, 7), (130, 255), (1000, 64), (5, 2048), (9, 7168), (2, 40000))]
    calls += [launches.rows(63, 1, 2), launches.rows(300000, 2, 8)]
    got, ours = launched(calls, tmp_path)
    assert len(ours) > 100 and ours - set().union(*got) == set()
