"""Host-only checks of distillation's workspace, of overlapping arguments and of how the operators are reached, without touching a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2509_11254_b200 import binding, build

    build.build_library()
    return binding.lib()


def test_distillation_workspace_is_bounded_in_entries(L):
    """Beside what the cross entropy of the same size holds and 8 bytes per token: the entries of a piece (16 bytes each) and its blocks of 32 rows and 32 columns, within a fixed size
    however many tokens there are and however long their lists."""
    a, b = C.c_size_t(), C.c_size_t()
    for grad in (0, 1):
        for T in (1 << 14, 1 << 17, 1 << 20, 1 << 24):
            for V in (40, 1000, 32000, 131072):
                for K in (1, 64, 1000, 1024):
                    assert L.psgd_distill_workspace(T, V, 64, K, grad, C.byref(a)) == 0 and L.psgd_xent_workspace(T, V, 64, grad, C.byref(b)) == 0
                    # (4 bytes per block of at most 2^32 logits, 4 per token of a piece, float32 sums of the weight gradient once there are several pieces, partial tiles)
                    assert a.value <= b.value + 8 * T + (1 << 30) + 4 * (1 << 22) + (1 << 27) + 4 * min(T, 1 << 25) + 4 * V * 64 + (1 << 26), (T, V, K, grad)
