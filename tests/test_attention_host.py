"""CPU-side checks of the attention's boundary: exports, the plain C header, argument checks before anything touches the GPU, the
tensor calls' refusals, and the arithmetic by which calls are cut (csrc/attention_selftest.cpp, under the sanitizers)."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2603_08343_amd as wht
from paper_2603_08343_amd import attention, build
from test_host_sanitizers import CSRC, SAN, _run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wht_attention.h")


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(wht_attention_\w+)\s*\(", text))
    lib = ctypes.CDLL(attention.library_path())
    assert names == set(attention.EXPORTS) and all(hasattr(lib, n) for n in names)


def test_statuses_have_strings():
    seen = {wht.wht_attention_status_string(s) for s in range(7)}
    assert len(seen) == 7 and "ok" in seen
    assert wht.wht_attention_status_string(99) == "unknown status"


def test_selftest_under_sanitizers(tmp_path):
    exe = str(tmp_path / "attention_san")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", *SAN, "-o", exe, os.path.join(CSRC, "attention_selftest.cpp")], check=True)
    assert "attention_selftest: ok" in _run(exe)


def test_header_is_plain_c_and_links(tmp_path):
    src = tmp_path / "use.c"
    src.write_text(r'''
#include <stdio.h>
#include "wht_attention.h"
int main(void) {
    wht_attention_rows_t r = {(void *)16, 512, 128}, none = {NULL, 0, 0};
    wht_attention_cache_t c = {(void *)16, (void *)16, 32768, 8192, 128, 4, 4, 64, 128};
    wht_attention_batch_t b = {(const int32_t *)16, (const int32_t *)16, NULL, 2, 3, 2};
    if (wht_attention_append(&none, &r, &none, &none, 3, 0, &c, &b, NULL, 0, 0, 0, 0, WHT_DTYPE_BF16, NULL) != WHT_ERR_NULL_PTR) return 1;
    if (wht_attention_append(&none, &r, &r, &none, 0, 0, &c, &b, NULL, 0, 0, 0, 0, WHT_DTYPE_BF16, NULL) != WHT_OK) return 2;
    size_t need = wht_attention_workspace_bytes(3, 3, 4, 4, 128, 1, 128, 0, WHT_DTYPE_BF16);
    if (need == 0) return 3;
    if (wht_attention_paged(&r, &r, NULL, 3, 4, &c, &b, NULL, 0, 1, 128, 1.0f, WHT_DTYPE_BF16, NULL, 0, NULL) != WHT_ERR_WORKSPACE) return 4;
    if (wht_attention_paged(&r, &r, NULL, 3, 4, &c, &b, NULL, 0, 1, 128, 1.0f, WHT_DTYPE_BF16, (void *)16, need - 1, NULL) != WHT_ERR_WORKSPACE) return 5;
    if (wht_attention_paged(&r, &r, NULL, 3, 4, &c, &b, NULL, 0, 1, 128, 1.0f, WHT_DTYPE_BF16, (void *)24, need, NULL) != WHT_ERR_MISALIGNED) return 6;
    if (wht_attention_paged(&r, &r, NULL, 0, 4, &c, &b, NULL, 0, 1, 128, 1.0f, WHT_DTYPE_BF16, NULL, 0, NULL) != WHT_OK) return 7;
    if (wht_attention_workspace_bytes(3, 3, 5, 4, 128, 1, 128, 0, WHT_DTYPE_BF16) != 0) return 8;
    printf("%s\n", wht_attention_status_string(WHT_OK));
    return 0;
}
''')
    exe = tmp_path / "use"
    libdir = os.path.dirname(attention.library_path())
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src),
                    "-L", libdir, "-l:libwht_attention.so", f"-Wl,-rpath,{libdir}"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", (out.returncode, out.stderr)


def test_missing_library_fails_loudly(monkeypatch):
    monkeypatch.setattr(attention, "_lib", None)
    monkeypatch.setattr(attention, "_LIB_PATH", "/nonexistent/libwht_attention.so")
    with pytest.raises(RuntimeError, match="no CPU or eager fallback"):
        attention.library()


@pytest.mark.skipif(torch.cuda.is_available(), reason="what happens without a GPU")
def test_no_cpu_path():
    p = torch.zeros(2, 4, 16, 64)
    q, i = torch.zeros(1, 4, 64), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(RuntimeError, match="needs an AMD GPU"):
        wht.wht_attention_paged(q, p, p, i, i[0])
    with pytest.raises(RuntimeError, match="needs an AMD GPU"):
        wht.wht_attention_append(q, q, q, p, p, i, i[0], None)


def test_rope_table():
    t = wht.wht_attention_rope_table(1000, 64, device="cpu")
    assert t.shape == (1000, 32, 2) and t.dtype == torch.float32
    angle = 999 * 10000.0 ** (-2.0 * 5 / 64)
    assert torch.equal(t[999, 5], torch.tensor([math.cos(angle), math.sin(angle)]))


@pytest.mark.parametrize("source", ["wht_attention.hip", "attention_device.h", "attention_plan.h", build.ATTENTION_HEADER])
def test_an_older_library_is_refused(source, monkeypatch):
    source = os.path.join(build.HERE, "csrc", source)
    real = os.path.getmtime
    build.ensure_built()
    monkeypatch.setattr(os.path, "getmtime", lambda f: real(source) - 1.0 if f == build.ATTENTION_LIB else real(f))
    with pytest.raises(RuntimeError, match="older than its source"):
        build.ensure_built()


def test_without_the_extension_module_calls_are_declined_after_one_warning(monkeypatch, recwarn):
    import sys
    monkeypatch.setitem(sys.modules, "paper_2603_08343_amd._attention_marshal", None)
    monkeypatch.delattr(wht, "_attention_marshal", raising=False)
    monkeypatch.setattr(attention, "_native_module", None)
    monkeypatch.setattr(attention, "_torch", lambda: torch)              # as if a GPU had been seen
    for _ in range(2):
        native = attention._native()
        assert native.append(*[None] * 12) is None and native.paged(*[None] * 15) is None
    assert [w.category for w in recwarn] == [RuntimeWarning]


@pytest.mark.parametrize("x,error", [(1 << 31, ValueError), (-(1 << 31) - 1, ValueError), ((1 << 32) + 1, ValueError), (1 << 64, ValueError), (2.5, ValueError),
                                     ("7", ValueError), (None, TypeError), ("x", TypeError), (math.nan, TypeError), (math.inf, TypeError)])
def test_numbers_that_do_not_fit_are_refused(x, error):
    """ctypes would cut them off: max_q = 2^32 + 1 would be 1."""
    with pytest.raises(error, match="max_q must be a whole number"):
        wht.wht_attention_workspace_bytes(3, 3, 4, 4, 128, x, 128, 0, 1)
    wide = (1 << 64) + 5 if x == 1 << 64 else x
    if error is TypeError or x == 1 << 64:
        with pytest.raises(error, match="max_length must be a whole number"):
            wht.wht_attention_workspace_bytes(3, 3, 4, 4, 128, 1, wide, 0, 1)


def test_whole_numbers_of_any_kind():
    want = wht.wht_attention_workspace_bytes(3, 3, 4, 4, 128, 2, 128, 0, 1)
    assert want > 0
    for kind in (np.int64, np.int32, torch.tensor, float):
        assert wht.wht_attention_workspace_bytes(3, 3, 4, 4, 128, kind(2), kind(128), kind(0), 1) == want


def test_assembly_that_writes_m0_says_so():
    """A register that an asm statement writes and does not name may hold a value of the compiler's."""
    statements = []
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        statements += [s for s in re.findall(r"asm volatile\((.*?)\);", text, flags=re.S) if re.search(r"s_mov_b32 m0", s)]
    assert len(statements) == 3
    for s in statements:
        assert '"m0"' in s.rsplit(":", 1)[1], s


@pytest.mark.parametrize("source", ["attention_query.cpp", "attention_plan.h", build.ATTENTION_HEADER])
def test_older_rules_are_refused(source, monkeypatch):
    source = os.path.join(build.HERE, "csrc", source)
    real = os.path.getmtime
    build.ensure_built()
    monkeypatch.setattr(os.path, "getmtime", lambda f: real(source) - 1.0 if f == build.ATTENTION_QUERY_LIB else real(f))
    with pytest.raises(RuntimeError, match="older than its source"):
        build.ensure_built()


def test_rope_table_of_an_odd_width_is_refused():
    """Its last pair would have one element, and the call would take it for a table one wider."""
    for rotary in (15, 63, -2):
        with pytest.raises(ValueError, match="rotary must be even"):
            wht.wht_attention_rope_table(10, rotary, device="cpu")
    assert wht.wht_attention_rope_table(10, 0, device="cpu").shape == (10, 0, 2)
