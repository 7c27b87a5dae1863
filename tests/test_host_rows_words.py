"""Row counts, statistics and results at the C entry points: alignment and overlaps are refused; nothing is launched."""
import ctypes

import paper_1801_10585_amd as scnn

P = ctypes.c_void_p
M = 1 << 20


def at(k, off=0):
    return P(k * M + off)


def linear_fwd(rows_dev=None, **k):
    L = scnn.load_library()
    a = {"x": at(1), "w": at(2), "bias": at(3), "residual": at(4), "out": at(5), "pre": at(6), "workspace": at(7), **k}
    return L.linear_fwd(0, a["x"], 10, rows_dev, 8, a["w"], a["bias"], 8, 1, a["residual"], a["out"], a["pre"], a["workspace"], M, None)


def linear_bwd(rows_dev=None):
    return scnn.load_library().linear_bwd(0, at(1), 10, rows_dev, 8, at(2), 8, 1, at(3), at(4), at(5), at(6), at(7), at(8), M, None)


def norm_fwd(rows_dev=None, mean=at(6), rstd=at(7)):
    return scnn.load_library().layer_norm_fwd(0, at(1), 10, rows_dev, 8, at(2), at(3), ctypes.c_double(1e-5), at(5), mean, rstd, None)


def norm_bwd(rows_dev=None, mean=at(4), rstd=at(5)):
    return scnn.load_library().layer_norm_bwd(0, at(1), at(2), 10, rows_dev, 8, at(3), mean, rstd, at(6), at(7), at(8), at(9), M, None)


def error():
    return scnn.load_library().scnn_last_error()


def test_a_misaligned_row_count():
    for call in (linear_fwd, linear_bwd, norm_fwd, norm_bwd):
        for off in (1, 2, 4):
            assert call(rows_dev=at(20, off)) == -1 and b"aligned" in error(), call


def test_a_row_count_inside_what_is_written():
    for call, outs in ((linear_fwd, (5, 6, 7)), (linear_bwd, (5, 6, 7, 8)), (norm_fwd, (5, 6, 7)), (norm_bwd, (6, 7, 8, 9))):
        for k in outs:
            for off in (0, 24):
                assert call(rows_dev=at(k, off)) == -1 and b"overlap" in error(), (call, k)


def test_misaligned_statistics_and_result():
    for call in (norm_fwd, norm_bwd):
        for off in (1, 2):
            assert call(mean=at(30, off)) == -1 and b"aligned" in error()
            assert call(rstd=at(30, off)) == -1 and b"aligned" in error()
    one = lambda t, v: (t * 1)(v)  # noqa: E731
    for off in (1, 2, 4):
        rc = scnn.load_library().grad_clip(1, one(P, M), None, one(ctypes.c_int64, 10), one(ctypes.c_int, 0), ctypes.c_double(1.0),
                                           at(40, off), at(50), M, None)
        assert rc == -1 and b"aligned" in error()
