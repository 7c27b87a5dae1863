"""Host-side refusals of group norm, dropout and the 8-bit layers (nothing is launched), and the generator's known answers."""
import ctypes

import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

P = ctypes.c_void_p
M = 1 << 20


def caller(f, good):
    def call(**at):
        args = list(good)
        for k, v in at.items():
            args[int(k[1:])] = v
        return f(*args)
    return call


def test_the_generators_known_answers():
    # (of the generator's publication: counter and key of zeros, of ones, of digits of pi)
    assert ref.philox((0,) * 4, (0,) * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 0xffffffff
    assert ref.philox((f,) * 4, (f,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert ref.philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_sample_offsets_refusals():
    L = scnn.load_library()
    # (ndim, batch, coords, rows, rows_dev, offsets, stream)
    call = caller(L.sample_offsets, [3, 4, P(M), 10, P(2 * M), P(3 * M), None])
    assert call(_0=1) == -1 and call(_0=4) == -1 and call(_1=0) == -1 and call(_3=-1) == -1 and call(_3=1 << 31) == -2
    assert call(_2=None) == -1 and call(_5=None) == -1
    assert call(_2=P(M + 2)) == -1 and call(_4=P(2 * M + 4)) == -1 and call(_5=P(3 * M + 4)) == -1
    for same in (P(M + 152), P(2 * M)):
        assert call(_5=same) == -1 and b"overlap" in L.scnn_last_error()


def test_group_norm_refusals():
    L = scnn.load_library()
    d = ctypes.c_double
    for query in (L.group_norm_fwd_workspace, L.group_norm_bwd_workspace):
        assert query(0, 10000, 4, 64, 8) > 256 and query(1, 0, 1, 1, 1) >= 256
        for bad in ((3, 10, 1, 8, 2), (0, -1, 1, 8, 2), (0, 1 << 31, 1, 8, 2), (0, 10, 0, 8, 2), (0, 10, 1, 0, 1), (0, 10, 1, 8, 0), (0, 10, 1, 8, 3),
                    (0, 10, 1, (1 << 24) + 8, 8), (0, 10, (1 << 30) + 1, 8, 8), (0, 1 << 30, 1, 1 << 20, 1)):
            assert query(*bad) == 0, bad
    # (dtype, x, rows, offsets, batch, channels, groups, gamma, beta, eps, act, out, mean, rstd, workspace, bytes, stream)
    good = [0, P(M), 10, P(2 * M), 2, 8, 4, P(3 * M), P(4 * M), d(1e-5), 1, P(5 * M), P(6 * M), P(7 * M), P(8 * M), M, None]
    fwd = caller(L.group_norm_fwd, good)
    assert fwd(_0=7) == -1 and fwd(_6=3) == -1 and fwd(_6=0) == -1 and fwd(_4=0) == -1 and fwd(_2=-1) == -1 and fwd(_10=4) == -1
    assert fwd(_9=d(-1.0)) == -1 and fwd(_9=d(float("nan"))) == -1 and fwd(_9=d(float("inf"))) == -1
    assert fwd(_3=None, _2=9) == -1 and b"samples" in L.scnn_last_error()  # (no offsets: equal samples)
    assert fwd(_1=None) == -1 and fwd(_11=None) == -1
    for i in (1, 7, 8, 11, 12, 13):
        assert fwd(**{f"_{i}": P(30 * M + 2)}) == -1 and b"aligned" in L.scnn_last_error()
    assert fwd(_3=P(30 * M + 4)) == -1
    assert fwd(_5=1024, _2=10000, _14=None) == -3 and fwd(_5=1024, _2=10000, _15=256) == -3 and fwd(_14=P(8 * M + 64)) == -3
    for out in (11, 12, 13):
        for i in (1, 3, 7, 8, 11, 12, 13):
            if i != out:
                assert fwd(**{f"_{out}": good[i]}) == -1 and b"overlap" in L.scnn_last_error()
    # (dtype, x, g, rows, offsets, batch, channels, groups, gamma, beta, mean, rstd, act, dx, dgamma, dbeta, workspace, bytes, stream)
    good = [1, P(M), P(2 * M), 10, P(3 * M), 2, 8, 4, P(4 * M), P(5 * M), P(6 * M), P(7 * M), 2, P(8 * M), P(9 * M), P(10 * M), P(11 * M), M, None]
    bwd = caller(L.group_norm_bwd, good)
    for i in (1, 2, 10, 11):
        assert bwd(**{f"_{i}": None}) == -1
    assert bwd(_12=-1) == -1 and bwd(_7=5) == -1 and bwd(_5=-1) == -1 and bwd(_17=100) == -3 and bwd(_16=P(11 * M + 8)) == -3
    assert bwd(_4=None, _3=11) == -1
    for out in (13, 14, 15, 16):
        for i in (1, 2, 4, 8, 9, 10, 11, 13, 14, 15):
            if i != out:
                assert bwd(**{f"_{out}": good[i]}) == -1 and b"overlap" in L.scnn_last_error()


def test_dropout_refusals():
    L = scnn.load_library()
    d, u = ctypes.c_double, ctypes.c_uint64
    # (dtype, x, rows, rows_dev, channels, p, seed, offset, rng, residual, out, stream)
    good = [2, P(M), 10, P(2 * M), 8, d(0.5), u(1), u(2), P(3 * M), P(4 * M), P(5 * M), None]
    fwd = caller(L.dropout_fwd, good)
    assert fwd(_0=3) == -1 and fwd(_2=-1) == -1 and fwd(_2=1 << 31) == -2 and fwd(_4=0) == -1 and fwd(_4=1 << 29) == -2
    for p in (-1e-9, 1.0000001, float("nan")):
        assert fwd(_5=d(p)) == -1
    assert fwd(_1=None) == -1 and fwd(_10=None) == -1
    for i in (1, 9, 10):
        assert fwd(**{f"_{i}": P(30 * M + 1)}) == -1 and b"aligned" in L.scnn_last_error()
    assert fwd(_3=P(30 * M + 4)) == -1 and fwd(_8=P(30 * M + 4)) == -1
    for where in (P(M + 2), P(4 * M + 2), P(2 * M), P(3 * M + 8)):  # beside x, beside the residual, on the count, on the seed
        assert fwd(_10=where) == -1 and b"overlap" in L.scnn_last_error()
    assert fwd(_2=0) == 0
    bwd = caller(L.dropout_bwd, good[:9] + [P(5 * M), None])
    assert bwd(_5=d(2.0)) == -1 and bwd(_9=None) == -1 and bwd(_1=None) == -1 and bwd(_9=P(M + 2)) == -1 and bwd(_2=0) == 0


def test_int8_refusals():
    L = scnn.load_library()
    assert [L.int8_row_bytes(c) for c in (1, 64, 65, 131008)] == [64, 64, 128, 131008]
    assert L.int8_row_bytes(0) == -1 and L.int8_row_bytes(131009) == -2 and L.int8_row_bytes(-5) == -1
    assert L.linear_int8_fwd_workspace(1, 0, 10, 100, 8) > 256
    for bad in ((3, 0, 10, 8, 8), (0, 0, -1, 8, 8), (0, 0, 10, 0, 8), (0, 0, 10, 8, 0), (0, 0, 1 << 31, 8, 8), (0, 1, 10, 131009, 8)):
        assert L.linear_int8_fwd_workspace(*bad) == 0, bad
    # (dtype, x, rows, rows_dev, channels, q, scale, stream)
    rows = caller(L.quantize_rows, [0, P(M), 10, P(2 * M), 100, P(3 * M), P(4 * M), None])
    assert rows(_0=5) == -1 and rows(_4=0) == -1 and rows(_4=131009) == -2 and rows(_1=None) == -1 and rows(_5=None) == -1 and rows(_6=None) == -1
    assert rows(_1=P(M + 2)) == -1 and rows(_5=P(3 * M + 8)) == -1 and rows(_6=P(4 * M + 2)) == -1 and rows(_3=P(2 * M + 4)) == -1
    for q in (P(M + 16), P(2 * M), P(4 * M - 1264)):
        assert rows(_5=q) == -1 and b"overlap" in L.scnn_last_error()
    assert rows(_2=0) == 0
    # (dtype, w, c_in, c_out, q, scale, stream)
    weight = caller(L.quantize_weight, [1, P(M), 100, 10, P(3 * M), P(4 * M), None])
    assert weight(_2=0) == -1 and weight(_3=0) == -1 and weight(_2=131009) == -2 and weight(_1=None) == -1 and weight(_4=None) == -1
    assert weight(_4=P(3 * M + 4)) == -1 and weight(_4=P(M)) == -1 and weight(_5=P(3 * M + 64)) == -1
    # (dtype, x, x_scale, rows, rows_dev, c_in, w, w_scale, bias, c_out, act, residual, out, workspace, bytes, stream)
    good = [1, P(M), P(2 * M), 10, P(3 * M), 100, P(4 * M), P(5 * M), P(6 * M), 8, 2, P(7 * M), P(8 * M), P(9 * M), M, None]
    fwd = caller(L.linear_int8_fwd, good)
    assert fwd(_0=-1) == -1 and fwd(_3=-1) == -1 and fwd(_5=0) == -1 and fwd(_5=131072) == -2 and fwd(_9=0) == -1 and fwd(_10=4) == -1
    for i in (1, 6, 7, 12):
        assert fwd(**{f"_{i}": None}) == -1
    assert fwd(_1=P(M + 8)) == -1 and b"16 bytes" in L.scnn_last_error()
    assert fwd(_6=P(4 * M + 8)) == -1 and fwd(_8=P(6 * M + 1)) == -1 and fwd(_11=P(7 * M + 1)) == -1 and fwd(_12=P(8 * M + 1)) == -1
    assert fwd(_2=P(2 * M + 2)) == -1 and fwd(_7=P(5 * M + 2)) == -1 and fwd(_4=P(3 * M + 4)) == -1
    assert fwd(_2=None, _13=None) == -3 and fwd(_2=None, _14=256) == -3
    for i in (1, 2, 4, 6, 7, 8):
        assert fwd(_12=good[i]) == -1 and b"overlap" in L.scnn_last_error()
    assert fwd(_12=P(7 * M + 2)) == -1  # beside the residual, not on it
    assert fwd(_2=None, _13=P(M)) == -1
    assert fwd(_3=0) == 0


def test_python_refusals():
    x = torch.ones((4, 6))
    for call in (lambda: scnn.group_norm_fwd(x, 2), lambda: scnn.group_norm_bwd(x, x, 2, None, None, torch.ones(1, 2), torch.ones(1, 2)),
                 lambda: scnn.dropout_fwd(x, 0.5), lambda: scnn.dropout_bwd(x, 0.5), lambda: scnn.quantize_rows(x),
                 lambda: scnn.quantize_weight(x), lambda: scnn.linear_int8_fwd(x, x.to(torch.int8), x[0]),
                 lambda: scnn.sample_offsets(x.to(torch.int32), 1)):
        with pytest.raises(ValueError):
            call()
    for query, sizes in ((scnn.group_norm_fwd_workspace, (10, 1, 8, 2)), (scnn.group_norm_bwd_workspace, (10, 1, 8, 2)),
                         (scnn.linear_int8_fwd_workspace, (10, 8, 8))):
        assert query(torch.bfloat16, *sizes) >= 256
        with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
            query(torch.float64, *sizes)
    with pytest.raises(scnn.ScnnError):
        scnn.group_norm_fwd_workspace(torch.float32, 10, 1, 8, 3)
    with pytest.raises(scnn.ScnnError):
        scnn.int8_row_bytes(1 << 20)
