"""CPU checks of the sizes that aal_fp8_matmul states in include/aal.h: the last ones that it takes pass
validation, the next ones do not."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, ALIGN = 1, 3


@pytest.fixture(scope="module")
def L():
    from paper_2609_24150_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libaal.so is not built (run __graft_entry__.build())")
    return _lib


def test_the_header_states_them():
    text = open(os.path.join(ROOT, "include", "aal.h")).read()
    doc = text[text.index("One operand of a product"):text.index("aal_status_t aal_fp8_matmul(")]
    assert "1 <= M, N <= 2^28, M * N < 2^37, 1 <= K < 2^24" in doc and re.search(r"at least K and below 2\^24", doc)


@pytest.mark.parametrize("M,N,K,ok", [
    (1 << 28, 100, 100_000, True), ((1 << 28) + 1, 100, 100_000, False), (100, 1 << 28, 100_000, True),
    (100, (1 << 28) + 1, 100_000, False), (1 << 19, 1 << 18, 100, False), (1, 1, (1 << 24) - 16, True),
    (1, 1, 1 << 24, False)])
def test_sizes(L, M, N, K, ok):
    """Nothing is launched: `c` is misaligned, which is checked behind the sizes and the operands."""
    ld = (K + 15) // 16 * 16
    a, b = (L.Fp8Operand(16, 16, ld, 1, 4, 0, 0, 1) for _ in range(2))
    st = L.lib().aal_fp8_matmul(C.byref(a), C.byref(b), M, N, K, 8, 0, None, 0, None)
    assert st == (ALIGN if ok else ARG), L.lib().aal_last_error()
    if not ok:
        assert L.lib().aal_fp8_matmul_workspace_bytes(M, N, K) == 0


def test_the_distance_of_rows(L):
    for ld, ok in (((1 << 24) - 16, True), (1 << 24, False)):
        a, b = (L.Fp8Operand(16, 16, d, 1, 4, 0, 0, 1) for d in (ld, 64))
        assert L.lib().aal_fp8_matmul(C.byref(a), C.byref(b), 4, 4, 64, 8, 0, None, 0, None) == (ALIGN if ok else ARG)
