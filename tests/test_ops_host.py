"""The host side of the head's operators without a GPU: refusals, work spaces, and launches (with a stand-in for the HIP
runtime, whose kernels do not run)."""
import ctypes

import pytest

import paper_1610_02496_amd as pk
from tests import fake_hip

EINVAL, ERANGE = pk.binding.SABER_EINVAL, pk.binding.SABER_ERANGE
P = 1 << 20   # some address; nothing below gets as far as using it


def message():
    return pk.load_library().saber_ops_last_error().decode()


def norm(x=P, x_stride=8, weight=None, bias=None, rows=4, cols=8, dtype=0, wtype=0, eps=1e-5, y=P, mean=P, rstd=P, q=None, scale=None):
    return pk.load_library().saber_layer_norm_forward(x, x_stride, weight, bias, rows, cols, dtype, wtype, eps, y, mean, rstd, q, scale, None)


@pytest.mark.parametrize("bad,code,word", [
    (dict(dtype=3), EINVAL, "type"), (dict(wtype=-1), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(cols=0), EINVAL, "columns"),
    (dict(cols=(1 << 20) + 1, x_stride=1 << 21), ERANGE, "limits"), (dict(rows=1 << 31), ERANGE, "limits"), (dict(x_stride=7), EINVAL, "apart"),
    (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"), (dict(x=None), EINVAL, "x is null"), (dict(y=None), EINVAL, "y is null"),
    (dict(x=P + 2), EINVAL, "aligned"), (dict(mean=None), EINVAL, "mean"), (dict(rstd=P + 1), EINVAL, "rstd"), (dict(q=P), EINVAL, "together"),
    (dict(scale=P), EINVAL, "together"), (dict(weight=P + 2), EINVAL, "weight"), (dict(bias=P + 1, wtype=2), EINVAL, "bias")])
def test_layer_norm_refuses(bad, code, word):
    assert norm(**bad) == code and word in message()


def test_layer_norm_backward_refuses():
    def call(dy=P, dy_stride=8, x=P, x_stride=8, q=None, scale=None, mean=P, rstd=P, weight=None, rows=4, cols=8, dtype=0, wtype=0, dx=P, dw=P, db=P,
             space=P, nbytes=1 << 20):
        return pk.load_library().saber_layer_norm_backward(dy, dy_stride, x, x_stride, q, scale, mean, rstd, weight, rows, cols, dtype, wtype, dx, dw, db,
                                                           space, nbytes, None)
    for bad, word in ((dict(q=P, scale=P), "not both"), (dict(x=None), "checkpoint"), (dict(x=None, q=P), "together"), (dict(dy=None), "dy"),
                      (dict(dy_stride=3), "apart"), (dict(space=None), "workspace"), (dict(nbytes=8), "work space"), (dict(dw=P + 2), "dweight"),
                      (dict(dx=P + 1), "dx"), (dict(mean=None), "mean")):
        assert call(**bad) == EINVAL and word in message(), bad
    n = ctypes.c_int64()
    assert pk.load_library().saber_layer_norm_backward_workspace(4, 0, ctypes.addressof(n)) == EINVAL
    assert pk.load_library().saber_layer_norm_backward_workspace(4, 8, None) == EINVAL
    for rows, cols in ((0, 5), (1, 1), (100, 1000), (1 << 30, 1 << 20)):
        assert pk.load_library().saber_layer_norm_backward_workspace(rows, cols, ctypes.addressof(n)) == 0
        assert n.value >= 8 * cols and n.value % (8 * cols) == 0


def test_checkpoints_refuse():
    L = pk.load_library()
    assert L.saber_checkpoint8_save(P, 7, 4, 8, 0, P, P, None) == EINVAL and "apart" in message()
    assert L.saber_checkpoint8_save(None, 8, 4, 8, 0, P, P, None) == EINVAL
    assert L.saber_checkpoint8_save(P, 8, 4, 8, 0, None, P, None) == EINVAL
    assert L.saber_checkpoint8_save(P, 8, 4, 8, 9, P, P, None) == EINVAL
    assert L.saber_checkpoint8_restore(P, None, 4, 8, 0, P, None) == EINVAL
    assert L.saber_checkpoint8_restore(P, P, 4, 0, 0, P, None) == EINVAL
    assert L.saber_checkpoint8_save(None, 8, 0, 8, 0, None, None, None) == 0     # no rows: nothing to do


def xent(forward, x=P, x_stride=64, w=P, w_stride=64, target=P, t64=1, rows=100, vocab=1000, cols=64, dtype=2, out=(P, P), space=P, nbytes=1 << 34, lse=P,
         dloss=P):
    n = ctypes.c_int64(nbytes)
    L = pk.load_library()
    if forward:
        rc = L.saber_linear_xent_forward(x, x_stride, w, w_stride, target, t64, rows, vocab, cols, dtype, out[0], out[1], space, ctypes.addressof(n), None)
    else:
        rc = L.saber_linear_xent_backward(dloss, x, x_stride, w, w_stride, target, t64, lse, rows, vocab, cols, dtype, out[0], out[1], space,
                                          ctypes.addressof(n), None)
    return rc, n.value


@pytest.mark.parametrize("forward", [True, False])
def test_cross_entropy_refuses(forward):
    for bad, code, word in ((dict(vocab=0), EINVAL, "vocabulary"), (dict(vocab=1 << 31), ERANGE, "vocabulary"), (dict(cols=0), EINVAL, "columns"),
                            (dict(dtype=7), EINVAL, "type"), (dict(x_stride=63), EINVAL, "apart"), (dict(w_stride=1), EINVAL, "apart"),
                            (dict(w=None), EINVAL, "weight"), (dict(x=None), EINVAL, "x is null"), (dict(target=None), EINVAL, "target"),
                            (dict(target=P + 4), EINVAL, "target"), (dict(space=P + 8), EINVAL, "256"), (dict(nbytes=16), EINVAL, "needed")):
        assert xent(forward, **bad)[0] == code and word in message(), bad
    if forward:
        assert xent(True, out=(None, P))[0] == EINVAL and xent(True, out=(P, None))[0] == EINVAL
    else:
        assert xent(False, lse=None)[0] == EINVAL and xent(False, dloss=None)[0] == EINVAL
        assert xent(False, out=(None, None))[0] == 0                            # nothing is wanted
    L = pk.load_library()
    assert (L.saber_linear_xent_forward if forward else L.saber_linear_xent_backward)(*([P, 64, P, 64, P, 1] if forward else [P, P, 64, P, 64, P, 1, P]),
                                                                                      100, 1000, 64, 2, P, P, P, None, None) == EINVAL


@pytest.mark.parametrize("forward", [True, False])
def test_work_space_is_bounded(forward):
    """A piece of the vocabulary at a time: the gradients' need does not grow with the vocabulary beyond what a piece takes, the
    forward pass' by two floats per row and 128 words."""
    small, large = (xent(forward, rows=8192, vocab=v, cols=1000, x_stride=1000, w_stride=1000, space=None)[1] for v in (1 << 20, 1 << 26))
    if forward:
        assert large <= 65 * small and large <= 8 * 8192 * (1 << 26) // 128 * 1.02
    else:
        assert large <= small * 1.01 and large < 1 << 30
    rc, unaligned = xent(forward, rows=8192, vocab=1 << 20, cols=777, x_stride=777, w_stride=777, space=None)
    assert rc == 0 and unaligned < 4 << 30


def test_launches_stay_within_the_limits(tmp_path):
    """Every launch over a range of shapes is one that the (stand-in) runtime accepts, and few rows take the kernel for few rows."""
    lib = fake_hip.build(tmp_path)
    fake_hip.run(lib, """
    L = pk.load_library()
    space = np.zeros(1 << 16, dtype=np.uint8)
    P = (space.ctypes.data + 255) // 256 * 256
    n = ctypes.c_int64()

    def xent(rows, vocab, cols, dtype, stride):
        for backward in (0, 1):
            head = [P] if backward else []
            args = head + [P, stride, P, stride, P, 0] + ([P] if backward else []) + [rows, vocab, cols, dtype, P, P]
            call = L.saber_linear_xent_backward if backward else L.saber_linear_xent_forward
            assert call(*args, None, ctypes.addressof(n), None) == 0, L.saber_ops_last_error()
            assert call(*args, P, ctypes.addressof(n), None) == 0, (rows, vocab, cols, dtype, L.saber_ops_last_error())

    for rows in (1, 16, 17, 64, 65, 300, 5000, 70000):
        for vocab in (1, 300, 30011, 141000):
            for cols, stride in ((1, 1), (64, 64), (777, 800), (1000, 1000), (9000, 9000)):
                for dtype in (0, 1, 2):
                    few = launches("score_few")[0]
                    xent(rows, vocab, cols, dtype, stride)
                    lds = rows * ((cols + 31) // 32 * 64 + 16) * (3 if dtype == 0 else 1)
                    assert (launches("score_few")[0] > few) == (rows <= 64 and lds <= 150 * 1024), (rows, vocab, cols, dtype, launches("score_few"), few)
    for rows in (1, 5, 4097, 1 << 22):
        for cols in (1, 512, 513, 1024, 1025, 2048, 4096, 8192, 8193, 100000):
            for dtype in (0, 1, 2):
                for held in (0, 1):
                    assert L.saber_layer_norm_forward(P, cols, P, P, rows, cols, dtype, 0, 1e-5, P, P, P, P if held else None, P if held else None, None) == 0, (rows, cols, dtype, L.saber_ops_last_error())
                    assert L.saber_layer_norm_backward_workspace(rows, cols, ctypes.addressof(n)) == 0
                    assert L.saber_layer_norm_backward(P, cols, None if held else P, cols, P if held else None, P if held else None, P, P, P, rows, cols, dtype,
                                                       0, P, P, P, P, n.value, None) == 0, L.saber_ops_last_error()
                assert L.saber_checkpoint8_save(P, cols, rows, cols, dtype, P, P, None) == 0, (rows, cols, dtype, L.saber_ops_last_error())
                assert L.saber_checkpoint8_restore(P, P, rows, cols, dtype, P, None) == 0, L.saber_ops_last_error()
    assert launches("norm_backward")[0] > 0 and launches("product_kernel")[0] > 0
    """)
