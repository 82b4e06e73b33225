"""CPU checks of the C entry points on top logits and logits processing: the
arguments that validation rejects, before anything touches a GPU, and the
exact C types."""
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
aal_status_t (*f2)(const void*, aal_dtype_t, int64_t, int32_t, int32_t, float, void*, int32_t*, float*,
                   hipStream_t) = aal_topk_logits;
size_t (*f3)(aal_layout_t, int64_t, int32_t, int32_t) = aal_topk_loss_workspace_bytes;
aal_status_t (*f4)(const void*, aal_dtype_t, const void*, aal_dtype_t, const int32_t*, const float*, aal_layout_t,
                   int64_t, int32_t, int32_t, int32_t, int32_t, float, float, aal_loss_weights_t, float*, float*,
                   float*, float*, float*, float*, int32_t*, void*, aal_dtype_t, const float*, uint32_t, void*, size_t,
                   hipStream_t) = aal_topk_loss_fwd_bwd;
aal_status_t (*f5)(const void*, aal_dtype_t, int64_t, int32_t, const aal_logits_rules_t*, void*,
                   hipStream_t) = aal_logits_process;
aal_status_t (*f6)(const void*, aal_dtype_t, const void*, aal_dtype_t, int64_t, int32_t, const aal_logits_rules_t*,
                   void*, hipStream_t) = aal_logits_process_bwd;
_Static_assert(AAL_TOPK_MAX == 512, "longest list");
_Static_assert(sizeof(aal_logits_rules_t) == 15 * 8, "rules layout");
'''


def test_signatures(lib, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "toplist.c"
    src.write_text('#include "aal.h"\n' + SIGNATURES)
    r = subprocess.run([cc, "-std=c11", "-Werror", "-Wall", "-fsyntax-only", f"-I{os.path.join(ROOT, 'include')}",
                        str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert C.sizeof(lib.LogitsRules) == 15 * 8


def test_workspace_bytes(lib):
    L = lib.lib()
    a = L.aal_topk_loss_workspace_bytes(0, 2048, 0, 7)
    assert a > 0 and a % 256 == 0 and L.aal_topk_loss_workspace_bytes(1, 2, 5, 7) > 0
    for bad in ((2, 1, 1, 1), (0, 0, 0, 7), (1, 2, 0, 7), (0, 2, 0, 65), (0, 2, 0, 0), (1, 1 << 30, 2, 1)):
        assert L.aal_topk_loss_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), 1), (dict(top=None), 1), (dict(ids=None), 1), (dict(rows=0), 1), (dict(rows=1 << 31), 1),
    (dict(V=0), 1), (dict(V=(1 << 30) + 1), 1), (dict(k=0), 1), (dict(k=101), 1), (dict(V=1000, k=513), 1),
    (dict(T=0.0), 1), (dict(T=float("nan")), 1), (dict(T=float("inf")), 1), (dict(dt=2), 2), (dict(dt=-1), 2),
    (dict(z=24), 3),
])
def test_topk_validation(lib, kw, code):
    a = dict(z=16, dt=0, rows=4, V=100, k=5, T=1.0, top=16, ids=16)
    a.update(kw)
    L = lib.lib()
    assert L.aal_topk_logits(a["z"], a["dt"], a["rows"], a["V"], a["k"], a["T"], a["top"], a["ids"], None,
                             None) == code
    assert L.aal_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", [
    (dict(zd=None), 1), (dict(top=None), 1), (dict(ids=None), 1), (dict(loss=None), 1), (dict(lay=2), 1),
    (dict(B=0), 1), (dict(S=0), 1), (dict(K=0), 1), (dict(K=65), 1), (dict(B=1 << 30, S=4), 1), (dict(V=0), 1),
    (dict(V=(1 << 19) + 1), 1), (dict(k=0), 1), (dict(k=101), 1), (dict(Td=0.0), 1), (dict(Tt=-1.0), 1),
    (dict(w=(0.0, float("nan"), 0.0, 0.0)), 1), (dict(w=(0.0, 0.0, 0.0, float("inf"))), 1), (dict(flags=4), 1),
    (dict(dt=3), 2), (dict(tdt=3), 2), (dict(grad=16, gdt=3), 2), (dict(zd=8), 3), (dict(grad=8), 3),
    (dict(ws=None), 4), (dict(ws=16), 3), (dict(wsb=100), 4),
])
def test_topk_loss_validation(lib, kw, code):
    a = dict(zd=16, dt=0, top=16, tdt=0, ids=16, lay=1, B=2, S=9, K=3, V=100, k=5, Td=1.0, Tt=1.0,
             w=(0.0, 0.0, 1.0, 0.0), loss=16, grad=None, gdt=0, flags=0, ws=256, wsb=1 << 40)
    a.update(kw)
    L = lib.lib()
    st = L.aal_topk_loss_fwd_bwd(a["zd"], a["dt"], a["top"], a["tdt"], a["ids"], None, a["lay"], a["B"], a["S"], a["K"],
                                 a["V"], a["k"], a["Td"], a["Tt"], lib.LossWeights(*a["w"]), a["loss"], None, None,
                                 None, None, None, None, a["grad"], a["gdt"], None, a["flags"], a["ws"], a["wsb"], None)
    assert st == code
    assert L.aal_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), 1), (dict(out=None), 1), (dict(no_rules=True), 1), (dict(rows=0), 1), (dict(V=0), 1),
    (dict(V=(1 << 24) + 1), 1), (dict(dt=9), 2), (dict(z=8), 3), (dict(out=8), 3),
    (dict(tokens=16), 1), (dict(tokens=16, hist_start=16), 1), (dict(hist_len=16), 1), (dict(repetition=16), 1),
    (dict(tokens=16, hist_start=16, hist_len=16, n_tokens=-1), 1), (dict(bias_ids=16), 1), (dict(bias_offsets=16), 1),
    (dict(bias_offsets=16, bias_ids=16, bias_values=16, n_bias=-1), 1), (dict(mask=16), 1), (dict(mask_row=16), 1),
    (dict(mask=16, n_masks=2), 1),
])
@pytest.mark.parametrize("backward", [False, True])
def test_process_validation(lib, kw, code, backward):
    a = dict(z=16, dt=0, rows=3, V=100, out=16)
    rules = lib.LogitsRules()
    for n, v in kw.items():
        if n in a:
            a[n] = v
        elif n != "no_rules":
            setattr(rules, n, v)
    r = None if kw.get("no_rules") else C.byref(rules)
    L = lib.lib()
    if backward:
        st = L.aal_logits_process_bwd(16, a["dt"], a["z"], a["dt"], a["rows"], a["V"], r, a["out"], None)
    else:
        st = L.aal_logits_process(a["z"], a["dt"], a["rows"], a["V"], r, a["out"], None)
    assert st == code
    assert L.aal_last_error().decode() != ""
