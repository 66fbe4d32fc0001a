"""Edges of the operators' range on the host side, without a GPU: empty batches, the largest sizes, what work space they ask for."""
import ctypes

import pytest

import paper_1610_02496_amd as pk
from tests import fake_hip


def test_no_product_of_an_empty_batch(tmp_path):
    """Without rows the gradients' products would have no steps at all: the weight's gradient is filled with zeros instead."""
    lib = fake_hip.build(tmp_path)
    fake_hip.run(lib, """
    L = pk.load_library()
    space = np.zeros(1 << 16, dtype=np.uint8)
    P = (space.ctypes.data + 255) // 256 * 256
    n = ctypes.c_int64()
    for vocab in (1, 300, 30011, 1 << 30):
        for cols in (1, 64, 777, 9000):
            for dtype in (0, 1, 2):
                for dx in (None, P):
                    args = [P, P, cols, P, cols, P, 0, P, 0, vocab, cols, dtype, dx, P]
                    assert L.saber_linear_xent_backward(*args, None, ctypes.addressof(n), None) == 0
                    zeros = launches("zeros_kernel")[0]
                    assert L.saber_linear_xent_backward(*args, P, ctypes.addressof(n), None) == 0, L.saber_ops_last_error()
                    assert launches("zeros_kernel")[0] == zeros + 1
    assert launches("product_kernel")[0] == 0
    """)


def need(backward, rows, vocab, cols, dtype, stride=None):
    n = ctypes.c_int64()
    L, P, s = pk.load_library(), 1 << 20, stride or cols
    if backward:
        rc = L.saber_linear_xent_backward(P, P, s, P, s, P, 1, P, rows, vocab, cols, dtype, P, P, None, ctypes.addressof(n), None)
    else:
        rc = L.saber_linear_xent_forward(P, s, P, s, P, 1, rows, vocab, cols, dtype, P, P, None, ctypes.addressof(n), None)
    assert rc == 0, L.saber_ops_last_error()
    return n.value


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,vocab,cols", [(64, 141_000, 1000), (2048, 60_000, 512), (300, 200_000, 2048), (8192, 141_000, 1000), (4096, 1 << 24, 777), (65, 1 << 28, 64)])
def test_work_space_of_every_type_is_bounded(rows, vocab, cols, dtype):
    """d of a piece and its packed words take 256 MB each at most; besides there are copies of the features (ten bytes a value at most)
    and partial sums of dx (of as many tiles as the CUs hold), forward a maximum and a sum per row and 64 words at most."""
    features, pad = rows * -(-cols // 8) * 8, 1 << 20
    assert need(True, rows, vocab, cols, dtype) <= 2 * (1 << 28) + 10 * features + max(4 * features, 1 << 27) + 8 * min(vocab, 1 << 20) + pad
    assert need(False, rows, vocab, cols, dtype) <= (1 << 28) + 4 * features + (rows + 16) * 8 * (vocab // 64 + 1) + 8 * min(vocab, 1 << 20) + pad


def test_binary32_work_space_is_smaller_than_large_logits():
    for rows, vocab, cols in ((2048, 60_000, 512), (4096, 100_000, 1024), (8192, 141_000, 1000)):
        for backward in (False, True):
            assert need(backward, rows, vocab, cols, 0) < 4 * rows * vocab


def test_the_largest_batches_are_refused_up_front_or_launched_whole(tmp_path):
    """Either every launch of a call stays within the runtime's limits (fewer than 2^32 threads), or nothing is launched at all."""
    lib = fake_hip.build(tmp_path)
    fake_hip.run(lib, """
    L = pk.load_library()
    space = np.zeros(1 << 16, dtype=np.uint8)
    P = (space.ctypes.data + 255) // 256 * 256
    n = ctypes.c_int64()
    refused = 0
    for rows in ((1 << 26) - 17, (1 << 26) - 16, (1 << 26) - 15, (1 << 26) - 1, 1 << 26, 1 << 25):
        for vocab, cols in ((1, 1), (300, 64), (70000, 1024), (300, 9000), (20, 1 << 18)):
            for dtype in (0, 1, 2):
                for backward in (0, 1):
                    args = ([P] if backward else []) + [P, cols, P, cols, P, 0] + ([P] if backward else []) + [rows, vocab, cols, dtype, P, P]
                    call = L.saber_linear_xent_backward if backward else L.saber_linear_xent_forward
                    before = launches("kernel")[0]
                    rc = call(*args, None, ctypes.addressof(n), None)
                    if rc == 0:
                        rc = call(*args, P, ctypes.addressof(n), None)
                        assert rc == 0, (rows, vocab, cols, dtype, backward, L.saber_ops_last_error())
                    else:
                        refused += 1
                        assert rc == pk.binding.SABER_ERANGE and launches("kernel")[0] == before
                    assert (rows <= (1 << 26) - 16) or rc != 0
                    assert not (rows <= (1 << 26) - 16 and cols <= 9000) or rc == 0, (rows, vocab, cols, dtype, backward, L.saber_ops_last_error())
    assert refused
    """)
