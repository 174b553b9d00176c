"""Operands that share memory where a call does not allow it are refused, wherever they begin (every call fails validation, so
no kernel is launched and the addresses are never read)."""
import os

import pytest

import paper_2606_10520_amd.unisvq as u

pytestmark = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")

OK, EINVAL = 0, -1
P, X, S, Y, W = (i << 24 for i in range(1, 6))  # 16 MB apart


def products(problems, M=4, xt=u.F16, yt=u.F16, ws=W, size=1 << 40):
    arr = (u.FourbitProblem * len(problems))(*problems)
    return u.load().unisvq_fourbit_gemm_batched(arr, len(problems), M, xt, yt, ws, size, None)


# 256 x 512: codes 64 KB and scales 2 KB; x of 4 tokens 4 KB (8 bits 2 KB), y of 16 bits 2 KB
@pytest.mark.parametrize("y", [P + 64, P + 66 * 1024 - 2, P - 2046, X + 2, X + 4094, X - 2046])
@pytest.mark.parametrize("other", [False, True])
def test_an_output_inside_an_input(y, other):
    """of its own problem, or of another one."""
    far = (256, 512, P + (1 << 23), X + (1 << 23), None, Y)
    one = (256, 512, P, X, None, Y + (1 << 20) if other else y)
    assert products([one, far[:5] + (y,)] if other else [one]) == EINVAL


@pytest.mark.parametrize("xt,M,y", [(u.I8, 4, X + 2046), (u.I8, 4, S + 14), (u.I8, 4, S - 2046), (u.I8, 500, S + 1998)])
def test_an_output_inside_scales_or_codes(xt, M, y):
    assert products([(256, 512, P, X, S, y)], M=M, xt=xt) == EINVAL


@pytest.mark.parametrize("yt,y", [(u.F16, Y + 2046), (u.F16, Y - 2046), (u.F32, Y + 4092), (u.F32, Y - 4092)])
def test_two_outputs(yt, y):
    assert products([(256, 512, P, X, None, Y), (256, 512, P, X, None, y)], yt=yt) == EINVAL


@pytest.mark.parametrize("xt", [u.F16, u.I8])
@pytest.mark.parametrize("name", ["packed", "x", "scales", "y"])
@pytest.mark.parametrize("end", ["first", "last"])
def test_a_workspace_that_an_operand_lies_in(xt, name, end):
    N, K, M = 1024, 8192, 100
    need = u.load().unisvq_fourbit_gemm_workspace_bytes(N, K, M, xt)
    assert need > 1 << 16
    size = {"packed": u.fourbit_bytes(N, K), "x": M * K * (1 if xt == u.I8 else 2), "scales": 4 * M, "y": 2 * M * N}[name]
    if name == "scales" and xt != u.I8:
        name, size = "x", 2 * M * K
    at = W + need - 16 if end == "last" else W - size + 16
    a = {"packed": P, "x": X, "scales": S if xt == u.I8 else None, "y": Y, **{name: at}}
    assert products([(N, K, a["packed"], a["x"], a["scales"], a["y"])], M=M, xt=xt, size=need) == EINVAL


def test_packing_in_place():
    lib = u.load()
    N, K = 256, 512
    for at in (X - 2048 * 33 + 16, X, X + 16 * 8191):
        assert lib.unisvq_fourbit_pack(N, K, X, S, at, None, None) == EINVAL
        assert lib.unisvq_fourbit_unpack(N, K, at, X, S, None) == EINVAL
        assert lib.unisvq_fourbit_quantize(N, K, X, u.F16, at, None) == EINVAL
    assert lib.unisvq_fourbit_pack(N, K, X, S, S + 2032, None, None) == EINVAL
    assert lib.unisvq_fourbit_pack(N, K, X, S, P, P + 4, None) == EINVAL
    assert lib.unisvq_fourbit_unpack(N, K, S + 2032, X, S, None) == EINVAL
    assert lib.unisvq_fourbit_unpack(N, K, P, X, X + 2, None) == EINVAL
    assert lib.unisvq_fourbit_quantize(N, K, X, u.F32, X + 4 * N * K - 16, None) == EINVAL
