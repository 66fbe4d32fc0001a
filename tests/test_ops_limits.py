"""Edges of the operators' range on the host side, without a GPU: empty batches, the largest sizes, what work space they ask for."""
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
