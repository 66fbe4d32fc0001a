"""The host side of the operators of a head that answers, without a GPU: refusals, work spaces, and launches (with a stand-in for the
HIP runtime, whose kernels do not run)."""
import ctypes

import pytest

import paper_1610_02496_amd as pk
from tests import fake_hip

EINVAL, ERANGE = pk.binding.SABER_EINVAL, pk.binding.SABER_ERANGE
P = 1 << 20   # some address; nothing below gets as far as using it


def message():
    return pk.load_library().saber_ops_last_error().decode()


def rms(x=P, x_stride=8, res=P, r_stride=8, weight=None, rows=4, cols=8, dtype=2, rtype=2, wtype=0, eps=1e-6, total=P, y=P, rstd=P, q=None, q_stride=16,
        scale=None):
    return pk.load_library().saber_rms_norm_forward(x, x_stride, res, r_stride, weight, rows, cols, dtype, rtype, wtype, eps, total, y, rstd, q, q_stride,
                                                    scale, None)


@pytest.mark.parametrize("bad,code,word", [
    (dict(dtype=3), EINVAL, "type"), (dict(wtype=-1), EINVAL, "type"), (dict(rtype=1), EINVAL, "stream"), (dict(rtype=5), EINVAL, "stream"), (dict(rows=-1), EINVAL, "rows"),
    (dict(cols=0), EINVAL, "columns"), (dict(cols=(1 << 20) + 1, x_stride=1 << 21), ERANGE, "limits"), (dict(rows=1 << 31), ERANGE, "limits"),
    (dict(x_stride=7), EINVAL, "apart"), (dict(r_stride=7), EINVAL, "apart"), (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"),
    (dict(x=None), EINVAL, "x is null"), (dict(y=None), EINVAL, "either"), (dict(q=P, scale=P), EINVAL, "either"), (dict(q=P), EINVAL, "together"),
    (dict(total=None), EINVAL, "together"), (dict(res=None), EINVAL, "together"), (dict(res=None, total=None, rtype=0), EINVAL, "without a residual"),
    (dict(x=P + 1), EINVAL, "aligned"), (dict(total=P + 1), EINVAL, "aligned"), (dict(rtype=0, res=P + 2), EINVAL, "aligned"), (dict(weight=P + 2), EINVAL, "weight"),
    (dict(rstd=P + 2), EINVAL, "rstd"), (dict(y=None, q=P, scale=P, q_stride=8), EINVAL, "16"), (dict(y=None, q=P + 8, scale=P), EINVAL, "16"),
    (dict(y=None, q=P, scale=P + 2), EINVAL, "scale"), (dict(y=None, q=P, scale=P, cols=17, x_stride=17, r_stride=17), EINVAL, "apart")])
def test_rms_norm_refuses(bad, code, word):
    assert rms(**bad) == code and word in message()


def test_rms_norm_backward_refuses():
    def call(dy=P, dy_stride=8, dsum=P, dsum_stride=8, s=P, s_stride=8, rstd=P, weight=None, rows=4, cols=8, dtype=2, rtype=0, wtype=0, dx=P, dres=P, dw=P,
             space=P, nbytes=1 << 20):
        return pk.load_library().saber_rms_norm_backward(dy, dy_stride, dsum, dsum_stride, s, s_stride, rstd, weight, rows, cols, dtype, rtype, wtype, dx, dres,
                                                         dw, space, nbytes, None)
    for bad, word in ((dict(dy=None), "dy"), (dict(s=None), "s is null"), (dict(rstd=None), "rstd"), (dict(dy_stride=3), "apart"), (dict(s_stride=3), "apart"),
                      (dict(dsum_stride=3), "apart"), (dict(dsum=P + 2), "dsum"), (dict(space=None), "workspace"), (dict(nbytes=8), "work space"),
                      (dict(dw=P + 2), "dweight"), (dict(dx=P + 1), "dx"), (dict(dres=P + 2), "dresidual"), (dict(rtype=1), "stream"), (dict(weight=P + 1), "weight")):
        assert call(**bad) == EINVAL and word in message(), bad
    n = ctypes.c_int64()
    L = pk.load_library()
    assert L.saber_rms_norm_backward_workspace(4, 0, ctypes.addressof(n)) == EINVAL
    assert L.saber_rms_norm_backward_workspace(4, 8, None) == EINVAL
    for rows, cols in ((0, 5), (1, 1), (100, 1000), (1 << 30, 1 << 20)):
        assert L.saber_rms_norm_backward_workspace(rows, cols, ctypes.addressof(n)) == 0
        assert n.value >= 4 * cols and n.value % (4 * cols) == 0


def test_rows_in_8_bits_refuse():
    L = pk.load_library()
    save = lambda x=P, xs=8, rows=4, cols=8, dtype=0, q=P, qs=16, scale=P: L.saber_rows8_save(x, xs, rows, cols, dtype, q, qs, scale, None)  # noqa: E731
    back = lambda q=P, qs=16, scale=P, rows=4, cols=8, dtype=0, x=P: L.saber_rows8_restore(q, qs, scale, rows, cols, dtype, x, None)  # noqa: E731
    for call in (save, back):
        for bad in (dict(x=None), dict(q=None), dict(scale=None), dict(qs=24), dict(qs=0), dict(q=P + 4), dict(x=P + 1), dict(scale=P + 1), dict(cols=0), dict(dtype=9)):
            assert call(**bad) == EINVAL, bad
        assert call(rows=0, q=None, x=None, scale=None) == 0
    assert save(xs=7) == EINVAL


def test_linear8_refuses():
    def call(x=P, xs=64, sx=P, w=P, ws=64, sw=P, rows=4, words=100, cols=64, dtype=2, out=P):
        return pk.load_library().saber_linear8(x, xs, sx, w, ws, sw, rows, words, cols, dtype, out, None)
    for bad, code, word in ((dict(cols=1 << 17, xs=1 << 17, ws=1 << 17), ERANGE, "columns"), (dict(words=0), EINVAL, "vocabulary"), (dict(words=1 << 31), ERANGE, "vocabulary"),
                            (dict(x=None), EINVAL, "x is null"), (dict(w=None), EINVAL, "weight"), (dict(sx=None), EINVAL, "x_scale"), (dict(sw=P + 1), EINVAL, "w_scale"),
                            (dict(xs=72), EINVAL, "16"), (dict(ws=48), EINVAL, "apart"), (dict(x=P + 8), EINVAL, "16"), (dict(out=P + 1), EINVAL, "out"),
                            (dict(xs=1 << 22), ERANGE, "stride"), (dict(ws=1 << 22), ERANGE, "stride"), (dict(rows=1 << 30, words=1 << 30), ERANGE, "rows"),
                            (dict(dtype=4), EINVAL, "type")):
        assert call(**bad) == code and word in message(), bad
    assert call(rows=0, x=None, out=None, sx=None) == 0


def test_sample_refuses():
    def call(logits=P, stride=100, rows=4, words=100, dtype=0, u=P, ts=None, t=1.0, ks=None, k64=0, k=0, ps=None, p=1.0, ms=None, m=0.0, word=P, share=P):
        return pk.load_library().saber_sample(logits, stride, rows, words, dtype, u, ts, t, ks, k64, k, ps, p, ms, m, word, share, None)
    nan = float("nan")
    for bad, code, text in ((dict(dtype=3), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(words=0), EINVAL, "words"), (dict(words=1 << 31, stride=1 << 31), ERANGE, "limits"),
                            (dict(rows=1 << 31), ERANGE, "limits"), (dict(stride=99), EINVAL, "apart"), (dict(t=-1.0), EINVAL, "temperature"), (dict(t=nan), EINVAL, "temperature"),
                            (dict(k=-1), EINVAL, "top_k"), (dict(p=1.01), EINVAL, "top_p"), (dict(p=nan), EINVAL, "top_p"), (dict(m=-0.1), EINVAL, "min_p"), (dict(m=nan), EINVAL, "min_p"),
                            (dict(logits=None), EINVAL, "logits"), (dict(u=None), EINVAL, "u is null"), (dict(ts=P + 1, t=nan), EINVAL, "temperatures"), (dict(ks=P + 4, k64=1), EINVAL, "top_ks"),
                            (dict(ps=P + 1, p=nan), EINVAL, "top_ps"), (dict(ms=P + 2, m=nan), EINVAL, "min_ps"), (dict(word=P + 4), EINVAL, "word"), (dict(share=None), EINVAL, "p is null")):
        assert call(**bad) == code and text in message(), bad
    assert call(rows=0, logits=None, u=None, word=None, share=None) == 0


def test_launches_stay_within_the_limits(tmp_path):
    """Every launch over a range of shapes is one that the (stand-in) runtime accepts."""
    lib = fake_hip.build(tmp_path)
    fake_hip.run(lib, """
    L = pk.load_library()
    space = np.zeros(1 << 16, dtype=np.uint8)
    P = (space.ctypes.data + 255) // 256 * 256
    n = ctypes.c_int64()
    up = lambda v: (v + 15) // 16 * 16
    for rows in (1, 5, 4097, 1 << 22, (1 << 31) - 1):
        for cols in (1, 512, 513, 1024, 1025, 2048, 4096, 8192, 8193, 100000, 1 << 20):
            for dtype, rtype in ((0, 0), (1, 1), (2, 2), (1, 0), (2, 0)):
                for q in (0, 1):
                    rc = L.saber_rms_norm_forward(P, cols, P, cols, P, rows, cols, dtype, rtype, 0, 1e-6, P, None if q else P, P, P if q else None, up(cols), P if q else None, None)
                    assert rc == 0, (rows, cols, dtype, L.saber_ops_last_error())
                assert L.saber_rms_norm_backward_workspace(rows, cols, ctypes.addressof(n)) == 0
                assert L.saber_rms_norm_backward(P, cols, P, cols, P, cols, P, P, rows, cols, dtype, rtype, 0, P, P, P, P, n.value, None) == 0, L.saber_ops_last_error()
                assert L.saber_rows8_save(P, cols, rows, cols, dtype, P, up(cols), P, None) == 0
                assert L.saber_rows8_restore(P, up(cols), P, rows, cols, dtype, P, None) == 0
    for rows in (1, 16, 17, 64, 65, 300, 5000, 70000, 1 << 24):
        for words in (1, 300, 30011, 141000, 1 << 24):
            for cols in (1, 64, 777, 1000, 131071):
                before = launches("kernel")[0]
                rc = L.saber_linear8(P, up(cols), P, P, up(cols), P, rows, words, cols, 2, P, None)
                tiles = -(-rows // 256) * -(-words // 256)
                assert rc == (0 if tiles < 1 << 24 else pk.binding.SABER_ERANGE), (rows, words, cols, L.saber_ops_last_error())
                assert (launches("kernel")[0] > before) == (rc == 0)
    for rows in (1, 300, 1 << 22, (1 << 31) - 1):
        for words in (1, 300, 8192, 8193, 141000, (1 << 31) - 1):
            for dtype in (0, 1, 2):
                assert L.saber_sample(P, words, rows, words, dtype, P, None, 1.0, None, 0, 5, None, 0.5, None, 0.1, P, P, None) == 0, L.saber_ops_last_error()
    assert launches("sample_kernel")[0] and launches("rms_backward")[0] and launches("product_kernel")[0]
    """)
