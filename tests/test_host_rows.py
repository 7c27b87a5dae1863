"""Host-side refusals of the layers on rows and of gradient clipping: nothing is launched."""
import ctypes

import pytest
import torch

import paper_1801_10585_amd as scnn

P = ctypes.c_void_p
BIG = 1 << 40


def test_linear_refusals():
    L = scnn.load_library()
    assert L.linear_fwd_workspace(0, 10, 8, 8) >= 256 and L.linear_fwd_workspace(2, 0, 1, 1) >= 256
    assert L.linear_bwd_workspace(1, 1000, 200, 200, 2) > L.linear_bwd_workspace(1, 1000, 200, 200, 0) >= 256
    assert L.linear_bwd_workspace(0, 0, 5, 3, 1) >= 256  # (no rows: the filter's gradient is still written)
    for bad in ((3, 10, 8, 8), (0, -1, 8, 8), (0, 10, 0, 8), (0, 10, 8, 0), (0, 1 << 31, 8, 8), (0, 10, (1 << 28) + 1, 8)):
        assert L.linear_fwd_workspace(*bad) == 0 and L.linear_bwd_workspace(*bad, 0) == 0
    assert L.linear_bwd_workspace(0, 10, 8, 8, 4) == 0 and b"activation" in L.scnn_last_error()
    # (dtype, x, rows, rows_dev, c_in, w, bias, c_out, act, residual, out, pre, workspace, bytes, stream)
    good = [0, P(1 << 20), 10, None, 8, P(2 << 20), P(3 << 20), 8, 1, P(4 << 20), P(5 << 20), P(6 << 20), P(7 << 20), 1 << 20, None]

    def fwd(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return L.linear_fwd(*args)

    assert fwd(_8=4) == -1 and fwd(_8=-1) == -1 and fwd(_0=9) == -1
    for i in (1, 5, 10):
        assert fwd(**{f"_{i}": None}) == -1
    for i in (1, 5, 6, 9, 10, 11):
        assert fwd(**{f"_{i}": P((30 << 20) + 2)}) == -1 and b"aligned" in L.scnn_last_error()
    assert fwd(_13=8) == -3 and fwd(_12=P((7 << 20) + 8)) == -3
    assert L.linear_fwd_workspace(0, 10, 1 << 14, 8) > 256  # (a split sum: needs its workspace)
    assert fwd(_4=1 << 14, _5=P(32 << 20), _12=None) == -3
    for i in (1, 5, 6, 11):
        assert fwd(_10=good[i]) == -1 and b"overlap" in L.scnn_last_error()
    assert fwd(_10=P((4 << 20) + 4)) == -1          # beside the residual, not on it
    assert fwd(_11=good[9]) == -1                    # pre on the residual
    assert fwd(_12=good[1]) == -1                    # workspace on an input
    assert fwd(_2=0) == 0                            # nothing to do
    # (dtype, x, rows, rows_dev, c_in, w, c_out, act, pre, g, dx, dw, dbias, workspace, bytes, stream)
    good = [0, P(1 << 20), 10, None, 8, P(2 << 20), 8, 1, P(3 << 20), P(4 << 20), P(5 << 20), P(6 << 20), P(7 << 20), P(8 << 20),
            1 << 20, None]

    def bwd(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return L.linear_bwd(*args)

    assert bwd(_7=5) == -1 and bwd(_9=None) == -1 and bwd(_1=None) == -1 and bwd(_5=None) == -1
    assert bwd(_8=None) == -1 and b"pre" in L.scnn_last_error()
    assert bwd(_14=16) == -3
    for i in (1, 5, 8, 9, 11, 12):
        assert bwd(_10=good[i]) == -1 and b"overlap" in L.scnn_last_error()


def test_layer_norm_refusals():
    L = scnn.load_library()
    d = ctypes.c_double
    # (dtype, x, rows, rows_dev, channels, gamma, beta, eps, out, mean, rstd, stream)
    good = [1, P(1 << 20), 10, None, 8, P(2 << 20), P(3 << 20), d(1e-5), P(4 << 20), P(5 << 20), P(6 << 20), None]

    def fwd(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return L.layer_norm_fwd(*args)

    assert fwd(_0=-1) == -1 and fwd(_2=-1) == -1 and fwd(_4=0) == -1 and fwd(_2=1 << 31) == -2 and fwd(_4=1 << 29) == -2
    assert fwd(_7=d(-1e-9)) == -1 and fwd(_7=d(float("nan"))) == -1 and fwd(_7=d(float("inf"))) == -1
    assert fwd(_1=None) == -1 and fwd(_8=None) == -1 and fwd(_1=P((1 << 20) + 1)) == -1
    for i in (1, 5, 6, 9):
        assert fwd(_8=good[i]) == -1 and b"overlap" in L.scnn_last_error()
    assert fwd(_2=0) == 0
    assert L.layer_norm_bwd_workspace(0, 100, 64) >= 512 and L.layer_norm_bwd_workspace(0, 100, 0) == 0
    assert L.layer_norm_bwd_workspace(5, 100, 64) == 0 and L.layer_norm_bwd_workspace(0, -1, 64) == 0
    # (dtype, x, g, rows, rows_dev, channels, gamma, mean, rstd, dx, dgamma, dbeta, workspace, bytes, stream)
    good = [0] + [P(i << 20) for i in (1, 2)] + [10, None, 8] + [P(i << 20) for i in (3, 4, 5, 6, 7, 8, 9)] + [1 << 20, None]

    def bwd(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return L.layer_norm_bwd(*args)

    for i in (1, 2, 7, 8):
        assert bwd(**{f"_{i}": None}) == -1
    assert bwd(_13=100) == -3 and bwd(_12=P((9 << 20) + 64)) == -3
    for i in (1, 2, 6, 7, 10):
        assert bwd(_9=good[i]) == -1 and b"overlap" in L.scnn_last_error()


def test_grad_clip_refusals():
    L = scnn.load_library()

    def clip(grads, outs, counts, types, max_norm=1.0, result=P(1 << 30), ws=P(2 << 30), nbytes=1 << 20):
        n = len(counts)
        arr = lambda v, t: None if v is None else (t * n)(*v)  # noqa: E731
        return L.grad_clip(n, arr(grads, P), arr(outs, P), arr(counts, ctypes.c_int64), arr(types, ctypes.c_int),
                           ctypes.c_double(max_norm), result, ws, nbytes, None)

    a, b = 1 << 20, 2 << 20
    assert clip([a, b], [a, b], [10, 10], [0, 0], max_norm=-1.0) == -1
    assert clip([a, b], [a, b], [10, 10], [0, 0], max_norm=float("nan")) == -1
    assert clip([a, b], [a, b], [10, 10], [0, 3]) == -1 and clip([a, b], [a, b], [10, -1], [0, 0]) == -1
    assert clip([a, b], [a, b], [BIG, 4 * BIG], [0, 0]) == -2
    assert clip([a, 0], [a, b], [10, 10], [0, 0]) == -1 and clip([a, b], [a, 0], [10, 10], [0, 0]) == -1
    assert clip(None, None, [10], [0]) == -1 and clip([a], [a], [10], None) == -1 and clip([a], [a], [10], [0], result=None) == -1
    assert clip([a + 2], [a + 2], [10], [0]) == -1 and clip([a], [a + 1], [10], [1]) == -1
    assert clip([a, b], [a, b], [10, 10], [0, 0], nbytes=8) == -3 and clip([a], [a], [10], [0], ws=P((2 << 30) + 8)) == -3
    # overlaps: the same tensor twice, ends that meet, an output on another gradient, at either end of it
    assert clip([a, a], [a, a], [10, 10], [0, 0]) == -1 and b"overlap" in L.scnn_last_error()
    assert clip([a, a + 36], [a, a + 36], [10, 10], [0, 0]) == -1
    assert clip([a, b], [b, a], [10, 10], [0, 0]) == -1
    assert clip([a, b], [a, a + 4096], [2000, 10], [0, 1]) == -1
    assert clip([a, b], [b + 36, b + 4096], [10, 10], [0, 0]) == -1
    assert clip([a, b], [b - 36, b + 4096], [10, 10], [0, 0]) == -1
    assert L.grad_clip_workspace(0, None) >= 256 and L.grad_clip_workspace(-1, None) == 0


def test_python_refusals():
    x = torch.ones((4, 6))
    with pytest.raises(ValueError):
        scnn.linear_fwd(x, torch.ones((6, 3)))
    with pytest.raises(ValueError):
        scnn.layer_norm_fwd(x)
    with pytest.raises(ValueError):
        scnn.clip_grad_norm([x], 1.0)
    with pytest.raises(ValueError):
        scnn.grad_norm([x])


def test_linear_in_place_is_for_the_residual_alone():
    # out on the residual is allowed; the same array as x, w or bias besides is not (other tiles still read those)
    L = scnn.load_library()
    for same in ("x", "w", "bias"):
        a = {"x": P(1 << 20), "w": P(2 << 20), "bias": P(3 << 20), "out": P(5 << 20)}
        a["out"] = a[same]
        rc = L.linear_fwd(0, a["x"], 8, None, 8, a["w"], a["bias"], 8, 0, a["out"], a["out"], None, P(7 << 20), 1 << 20, None)
        assert rc == -1 and b"overlap" in L.scnn_last_error(), same


def test_grad_clip_result_apart_from_the_workspace():
    L = scnn.load_library()
    g, count, kind = (P * 1)(1 << 20), (ctypes.c_int64 * 1)(10), (ctypes.c_int * 1)(0)
    for result, ws in ((2 << 30, 2 << 30), ((2 << 30) + 8, 2 << 30), (1 << 20, 2 << 30), ((1 << 20) + 32, 2 << 30),
                       (1 << 30, 1 << 20)):  # on the workspace, inside it, on a gradient, on its end; the workspace on one
        rc = L.grad_clip(1, g, None, count, kind, ctypes.c_double(1.0), P(result), P(ws), 1 << 20, None)
        assert rc == -1 and b"overlap" in L.scnn_last_error(), (result, ws)


def test_workspace_queries_refuse_other_types():
    for query, sizes in ((scnn.linear_fwd_workspace, (10, 8, 8)), (scnn.linear_bwd_workspace, (10, 8, 8)),
                         (scnn.layer_norm_bwd_workspace, (10, 8))):
        assert query(torch.bfloat16, *sizes) >= 256
        with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
            query(torch.float64, *sizes)
