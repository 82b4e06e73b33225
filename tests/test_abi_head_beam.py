"""CPU checks of the C entry points of the 8-bit head and of beam search: the
arguments that validation rejects, before anything touches a GPU, and the exact C types."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_24150_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libaal.so is not built (run __graft_entry__.build())")
    return _lib


SIGNATURES = '''
aal_status_t (*f1)(const void*, aal_dtype_t, int64_t, int64_t, int64_t, aal_fp8_t, aal_scale_t, int32_t, void*, int64_t,
                   void*, void*, int64_t, void*, hipStream_t) = aal_fp8_quantize;
size_t (*f2)(int64_t, int64_t, int64_t) = aal_fp8_matmul_workspace_bytes;
aal_status_t (*f3)(const aal_fp8_operand_t*, const aal_fp8_operand_t*, int64_t, int64_t, int64_t, void*, aal_dtype_t,
                   void*, size_t, hipStream_t) = aal_fp8_matmul;
size_t (*f4)(aal_dtype_t, int64_t, int32_t, int32_t, int32_t) = aal_beam_select_workspace_bytes;
aal_status_t (*f5)(const void*, aal_dtype_t, int64_t, int32_t, int32_t, int32_t, float, const float*, const uint8_t*,
                   const int32_t*, float, int32_t, int32_t, const aal_beam_out_t*, void*, size_t,
                   hipStream_t) = aal_beam_select;
aal_status_t (*f6)(const aal_beam_state_t*, int32_t, int64_t, int32_t, int32_t, const int32_t*,
                   hipStream_t) = aal_beam_reorder;
_Static_assert(sizeof(aal_fp8_operand_t) == 56, "operand layout");
_Static_assert(sizeof(aal_beam_out_t) == 48, "outputs layout");
_Static_assert(sizeof(aal_beam_state_t) == 80, "state layout");
_Static_assert(AAL_FP8_BLOCK == 128 && AAL_BEAM_MAX == 64 && AAL_BEAM_SELECT_MAX == 128, "constants");
'''


def test_signatures(lib, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "head_beam.c"
    src.write_text('#include "aal.h"\n' + SIGNATURES)
    r = subprocess.run([cc, "-std=c11", "-Werror", "-Wall", "-fsyntax-only", f"-I{os.path.join(ROOT, 'include')}",
                        str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert C.sizeof(lib.Fp8Operand) == 56 and C.sizeof(lib.BeamOut) == 48 and C.sizeof(lib.BeamState) == 80


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), 1), (dict(q=None, s=None), 1), (dict(s=None), 1), (dict(q=None), 1), (dict(qt=16), 1), (dict(st=16), 1),
    (dict(rows=0), 1), (dict(rows=1 << 31), 1), (dict(cols=0), 1), (dict(cols=(1 << 30) + 1, ld=1 << 31, ld_q=1 << 31), 1),
    (dict(ld=99), 1), (dict(block=2), 1), (dict(ld_q=96), 1), (dict(qt=16, st=16, ld_qt=0), 1), (dict(dt=2), 2),
    (dict(fmt=2), 2), (dict(sc=-1), 2), (dict(x=17), 3), (dict(q=24), 3), (dict(ld_q=120), 3),
    (dict(qt=16, st=16, ld_qt=40), 3), (dict(s=18), 3),
])
def test_quantize_validation(lib, kw, code):
    a = dict(x=16, dt=0, rows=4, cols=100, ld=100, fmt=0, sc=0, block=1, q=16, ld_q=112, s=16, qt=None, ld_qt=16, st=None)
    a.update(kw)
    L = lib.lib()
    assert L.aal_fp8_quantize(a["x"], a["dt"], a["rows"], a["cols"], a["ld"], a["fmt"], a["sc"], a["block"], a["q"],
                              a["ld_q"], a["s"], a["qt"], a["ld_qt"], a["st"], None) == code
    assert L.aal_last_error().decode() != ""


def test_matmul_workspace(lib):
    L = lib.lib()
    assert L.aal_fp8_matmul_workspace_bytes(8192, 128256, 4096) == 0
    n = L.aal_fp8_matmul_workspace_bytes(7, 4096, 128256)
    assert n > 0 and n % 256 == 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 29, 1, 1), (1, 1, 1 << 24), (1 << 20, 1 << 20, 1)):
        assert L.aal_fp8_matmul_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(c=None), 1), (dict(a=None), 1), (dict(b=None), 1), (dict(M=0), 1), (dict(N=1 << 29), 1), (dict(K=0), 1),
    (dict(K=1 << 24), 1), (dict(M=1 << 20, N=1 << 20), 1), (dict(values=None), 1), (dict(scale=None), 1),
    (dict(block_rows=64), 1), (dict(ld=48), 1), (dict(ld=1 << 24), 1), (dict(format=2), 2), (dict(scale_type=2), 2),
    (dict(scale_type=1), 2), (dict(dt=5), 2), (dict(values=24), 3), (dict(ld=72), 3), (dict(scale=18), 3), (dict(c=8), 3),
    (dict(K=128256, ld=128256, ld_b=128256), 4), (dict(K=128256, ld=128256, ld_b=128256, ws=16, wsb=1 << 40), 3),
    (dict(K=128256, ld=128256, ld_b=128256, ws=256, wsb=64), 4),
])
def test_matmul_validation(lib, kw, code):
    a = dict(M=4, N=100, K=64, c=16, dt=0, ws=None, wsb=0)
    oa, ob = (lib.Fp8Operand(16, 16, 64, 1, 4, 0, 0, 1) for _ in range(2))
    ob.ld = kw.get("ld_b", 64)
    for n, v in kw.items():
        if n in a:
            a[n] = v
        elif n in dict(lib.Fp8Operand._fields_):
            setattr(oa, n, v)
    L = lib.lib()
    st = L.aal_fp8_matmul(None if kw.get("a", 1) is None else C.byref(oa), None if kw.get("b", 1) is None else C.byref(ob),
                          a["M"], a["N"], a["K"], a["c"], a["dt"], a["ws"], a["wsb"], None)
    assert st == code
    assert L.aal_last_error().decode() != ""


def test_beam_workspace(lib):
    L = lib.lib()
    n = L.aal_beam_select_workspace_bytes(0, 64, 8, 128256, 16)
    assert n > 0 and n % 256 == 0
    for bad in ((2, 1, 1, 10, 1), (0, 0, 1, 10, 1), (0, 1, 65, 10, 1), (0, 1, 1, 0, 1), (0, 1, 1, (1 << 18) + 1, 1),
                (0, 1, 1, 10, 11), (0, 1, 4, 1000, 129), (0, 1 << 31, 1, 10, 1)):
        assert L.aal_beam_select_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), 1), (dict(scores=None), 1), (dict(no_out=True), 1), (dict(parents=None), 1), (dict(tokens=None), 1),
    (dict(B=0), 1), (dict(W=0), 1), (dict(W=65), 1), (dict(V=0), 1), (dict(V=(1 << 18) + 1), 1), (dict(n=0), 1),
    (dict(n=129), 1), (dict(B=1 << 30, W=2), 1), (dict(T=0.0), 1), (dict(T=float("nan")), 1), (dict(alpha=float("inf")), 1),
    (dict(alpha=1.0), 1), (dict(dt=7), 2), (dict(z=24), 3), (dict(ws=None), 4), (dict(ws=16), 3), (dict(wsb=10), 4),
])
def test_select_validation(lib, kw, code):
    a = dict(z=16, dt=0, B=2, W=3, V=1000, n=5, T=1.0, scores=16, lengths=None, alpha=0.0, ws=256, wsb=1 << 40)
    out = lib.BeamOut(None, None, 16, 16, None, None)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        elif k != "no_out":
            setattr(out, k, v)
    L = lib.lib()
    st = L.aal_beam_select(a["z"], a["dt"], a["B"], a["W"], a["V"], a["n"], a["T"], a["scores"], None, a["lengths"],
                           a["alpha"], -1, 0, None if kw.get("no_out") else C.byref(out), a["ws"], a["wsb"], None)
    assert st == code
    assert L.aal_last_error().decode() != ""


@pytest.mark.parametrize("kw", [
    dict(n_states=-1), dict(states=None), dict(parents=None), dict(B=0), dict(W=0), dict(n=0), dict(n=129),
    dict(B=1 << 30), dict(n=3, dst=None), dict(n=80, W=80, dst=None), dict(src=None), dict(segments=-1),
    dict(segment_bytes=-1), dict(segments=1 << 30, segment_bytes=1 << 30), dict(src_beam=1 << 50), dict(dst_segment=-(1 << 50)),
])
def test_reorder_validation(lib, kw):
    a = dict(states=1, n_states=1, B=2, W=4, n=4, parents=16)
    table = (lib.BeamState * 1)()
    table[0] = lib.BeamState(16, 4096, 256, 64, 0, 256, 64, 0, 1, 64)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            setattr(table[0], k, v)
    L = lib.lib()
    st = L.aal_beam_reorder(table if a["states"] else None, a["n_states"], a["B"], a["W"], a["n"], a["parents"], None)
    assert st == 1
    assert L.aal_last_error().decode() != ""


def test_reorder_of_nothing(lib):
    """No states, or states without a byte: nothing is launched (this runs without a GPU)."""
    L = lib.lib()
    assert L.aal_beam_reorder(None, 0, 1, 1, 1, 16, None) == 0
    table = (lib.BeamState * 2)(lib.BeamState(None, None, 0, 0, 0, 0, 0, 0, 0, 16), lib.BeamState(16, None, 0, 0, 0, 0, 0, 0, 4, 0))
    assert L.aal_beam_reorder(table, 2, 1, 4, 4, 16, None) in (0, 5)  # 5: the runtime, asked for its last error, has no device
