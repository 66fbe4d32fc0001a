"""Arguments of the operators that answer, as the torch entry points pass them on, without a GPU (in a process of its own: torch is imported before
the library); work spaces around the choice of a kernel's variant."""
from tests import fake_hip
from tests.test_ops_runtime import run

HEAD = """
import torch
import paper_1610_02496_amd as pk
from paper_1610_02496_amd import ops
L = pk.load_library()
"""


def test_top_k_of_any_size():
    """Whole numbers beyond 64 bits are not wrapped: below zero they are refused as -1 is, far above they are all words."""
    p = run(HEAD + """
P = 1 << 20
for k in (-1, -5, -(1 << 63), -(1 << 63) - 1, -(1 << 64), -(1 << 64) + 5, -(1 << 100)):
    values, number = ops._limit("top_k", k, (4,), None, (torch.int32, torch.int64))
    rc = L.saber_sample(P, 100, 4, 100, 0, P, None, 1.0, None, 0, number, None, 1.0, None, 0.0, P, P, None)
    assert values is None and rc == pk.binding.SABER_EINVAL and b"top_k" in L.saber_ops_last_error(), (k, number, rc)
for k in (0, 7, (1 << 62) - 1):
    assert ops._limit("top_k", k, (4,), None, (torch.int32, torch.int64)) == (None, k)
assert ops._limit("top_k", 1 << 64, (4,), None, (torch.int32, torch.int64))[1] >= 1 << 31
print("passed")
""")
    assert p.returncode == 0 and "passed" in p.stdout, p.stdout


def test_work_space_of_the_norm_suffices_for_either_variant(tmp_path):
    """The work space is asked for by sizes alone, the variant depends on the stream's type as well."""
    fake_hip.run(fake_hip.build(tmp_path), """
    L = pk.load_library()
    space = np.zeros(1 << 16, dtype=np.uint8)
    P = (space.ctypes.data + 255) // 256 * 256
    n = ctypes.c_int64()
    for rows in (1, 5, 1023, 1025, 4097, 23999, 39999, 40000, 65536, 1 << 24):
        for cols in (1, 1024, 1025, 1599, 1600, 2048, 2049):
            for dtype, rtype in ((0, 0), (1, 1), (2, 2), (1, 0), (2, 0)):
                assert L.saber_rms_norm_backward_workspace(rows, cols, ctypes.addressof(n)) == 0
                assert L.saber_rms_norm_backward(P, cols, P, cols, P, cols, P, P, rows, cols, dtype, rtype, 0, P, P, P, P, n.value, None) == 0, (rows, cols, L.saber_ops_last_error())
    """)
