"""CPU-side checks of the cache in 4 bits and of rotary positions: exports, the plain C headers, argument checks before anything touches the GPU, and
the definition that the GPU tests compare with, on numbers worked out by hand."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import attention4_check as check
import paper_2603_08343_amd as wht
from paper_2603_08343_amd import attention4, build, rotary
from test_host_sanitizers import CSRC, SAN, _run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("header,exports", [("wht_attention4.h", attention4.EXPORTS), ("wht_rotary.h", attention4.ROTARY_EXPORTS)])
def test_library_exports_every_declared_symbol(header, exports):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    names = set(re.findall(r"\b(wht_\w+)\s*\(", text))
    lib = ctypes.CDLL(attention4.library_path())
    assert names == set(exports) and all(hasattr(lib, n) for n in names)


@pytest.mark.parametrize("name", [wht.wht_attention4_status_string, wht.wht_rotary_status_string])
def test_statuses_have_strings(name):
    known = {s for s in range(7)} - ({5} if name is wht.wht_rotary_status_string else set())
    assert len({name(s) for s in known}) == len(known) and name(0) == "ok" and name(99) == "unknown status"


def test_headers_are_plain_c_and_arguments_are_checked(tmp_path):
    src = tmp_path / "use.c"
    src.write_text(r'''
#include <stdio.h>
#include "wht_attention4.h"
#define EXPECT(want, call) do { int got = (call); if (got != (want)) { printf("line %d: %d\n", __LINE__, got); return 1; } } while (0)
static wht_attention_rows_t r = {(void *)16, 512, 128}, q8 = {(void *)16, 1024, 128}, none = {NULL, 0, 0};
static wht_attention_cache4_t good = {(void *)16, (void *)16, (uint8_t *)1, (uint8_t *)1, 16384, 4096, 64, 1024, 256, 4, 4, 4, 64, 128}, c;
static wht_attention_batch_t b = {(const int32_t *)16, (const int32_t *)16, NULL, 2, 3, 2};
static uint8_t axes[64];
static int append(const wht_attention_rows_t *q, int64_t T, int rotary, const int32_t *positions, int count, int dtype) {
    return wht_attention_append4(q, &r, &r, q, &none, &none, T, q->data ? 4 : 0, &c, &b, rotary ? (const float *)16 : NULL, 100, rotary, 0, 0, positions, count, axes, 1, dtype, NULL);
}
static int paged(int64_t T, int heads, int64_t length, float scale, void *ws, size_t bytes) {
    return wht_attention_paged4(&q8, &q8, NULL, T, heads, &c, &b, NULL, 0, 1, length, scale, 1, WHT_DTYPE_BF16, ws, bytes, NULL);
}
static int rotate(int D, int rotary, int count, const uint8_t *pairs, int64_t T) {
    wht_attention_rows_t x = {(void *)16, 4096, 256};
    return wht_rotary_rotate(&x, &x, T, 4, D, (const float *)16, 10, rotary, 0, count > 1 ? (const int32_t *)16 : NULL, count, pairs, 0, WHT_DTYPE_BF16, NULL);
}
int main(void) {
    size_t need = wht_attention4_workspace_bytes(3, 3, 8, 4, 128, 1, 1 << 20, 0, WHT_DTYPE_BF16);
    const int32_t *at = (const int32_t *)16;
    c = good;
    EXPECT(WHT_OK, append(&r, 0, 64, at, 3, WHT_DTYPE_BF16));
    EXPECT(WHT_OK, append(&none, 0, 0, NULL, 1, WHT_DTYPE_F32));
    EXPECT(WHT_ERR_BAD_DTYPE, append(&r, 0, 0, NULL, 1, 7));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, -1, 0, NULL, 1, WHT_DTYPE_BF16));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 24, at, 3, WHT_DTYPE_BF16));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 144, at, 3, WHT_DTYPE_BF16));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 64, at, 0, WHT_DTYPE_BF16));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 64, at, 5, WHT_DTYPE_BF16));
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 64, NULL, 2, WHT_DTYPE_BF16));
    axes[31] = 3;
    EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 64, at, 3, WHT_DTYPE_BF16));
    EXPECT(WHT_OK, append(&r, 0, 48, at, 3, WHT_DTYPE_BF16));
    axes[31] = 0;
    EXPECT(WHT_ERR_NULL_PTR, wht_attention_append4(&none, &r, &r, &none, &r, &none, 0, 0, &c, &b, NULL, 0, 0, 0, 0, NULL, 1, NULL, 1, WHT_DTYPE_BF16, NULL));
    EXPECT(WHT_ERR_NULL_PTR, wht_attention_append4(&none, &r, &none, &none, &none, &none, 0, 0, &c, &b, NULL, 0, 0, 0, 0, NULL, 1, NULL, 1, WHT_DTYPE_BF16, NULL));
    c.k_scales = NULL; EXPECT(WHT_ERR_NULL_PTR, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.head_dim = 32; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.page_size = 48; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.token_stride = 48; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.scale_token_stride = 3; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.page_stride = (int64_t)1 << 32; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.scale_page_stride = (int64_t)1 << 32; EXPECT(WHT_ERR_BAD_DIM, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.head_stride = 4100; EXPECT(WHT_ERR_MISALIGNED, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.k = (void *)24; EXPECT(WHT_ERR_MISALIGNED, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    c.page_stride = 4096; EXPECT(WHT_ERR_MISALIGNED, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16));            /* written pages overlap */
    EXPECT(WHT_OK, paged(0, 8, 128, 1.0f, NULL, 0)); c = good;                                              /* read ones may */
    c.scale_page_stride = 256; EXPECT(WHT_ERR_MISALIGNED, append(&r, 0, 0, NULL, 1, WHT_DTYPE_BF16)); c = good;
    EXPECT(WHT_ERR_WORKSPACE, paged(3, 8, 1 << 20, 1.0f, NULL, 0));
    EXPECT(WHT_ERR_WORKSPACE, paged(3, 8, 1 << 20, 1.0f, (void *)16, need - 1));
    EXPECT(WHT_ERR_MISALIGNED, paged(3, 8, 1 << 20, 1.0f, (void *)24, need));
    EXPECT(WHT_ERR_BAD_DIM, paged(3, 7, 128, 1.0f, (void *)16, need));
    EXPECT(WHT_ERR_BAD_DIM, paged(3, 8, 128, 0.0f, (void *)16, need));
    EXPECT(WHT_ERR_BAD_DIM, paged(3, 8, 128, 3e38f, (void *)16, need));
    EXPECT(WHT_ERR_BAD_DIM, paged(3, 8, -1, 1.0f, (void *)16, need));
    EXPECT(0, (int)wht_attention4_workspace_bytes(3, 3, 5, 4, 128, 1, 128, 0, WHT_DTYPE_BF16));
    EXPECT(WHT_OK, rotate(128, 128, 3, axes, 0));
    EXPECT(WHT_OK, rotate(256, 256, 1, NULL, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(120, 64, 1, NULL, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(272, 64, 1, NULL, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 0, 1, NULL, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 80, 1, NULL, 0));
    axes[0] = 2;
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 64, 2, axes, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 64, 1, axes, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 64, 5, NULL, 0));
    EXPECT(WHT_ERR_BAD_DIM, rotate(64, 64, 1, NULL, ((int64_t)1 << 30) + 1));
    EXPECT(WHT_ERR_NULL_PTR, wht_rotary_rotate(&r, &r, 0, 4, 64, NULL, 10, 64, 0, NULL, 1, NULL, 0, WHT_DTYPE_BF16, NULL));
    printf("%s\n", wht_attention4_status_string(WHT_OK));
    return 0;
}
''')
    exe = tmp_path / "use"
    libdir = os.path.dirname(attention4.library_path())
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src),
                    "-L", libdir, "-l:libwht_attention4.so", f"-Wl,-rpath,{libdir}"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", (out.returncode, out.stdout, out.stderr)


def test_missing_library_fails_loudly(monkeypatch):
    monkeypatch.setattr(attention4, "_lib", None)
    monkeypatch.setattr(attention4, "_LIB_PATH", "/nonexistent/libwht_attention4.so")
    with pytest.raises(RuntimeError, match="no CPU or eager fallback"):
        attention4.library()


@pytest.mark.skipif(torch.cuda.is_available(), reason="what happens without a GPU")
def test_no_cpu_path():
    p, s = torch.zeros(2, 4, 16, 32, dtype=torch.uint8), torch.zeros(2, 4, 16, 2, dtype=torch.uint8)
    q, i = torch.zeros(1, 4, 64), torch.zeros(1, 1, dtype=torch.int32)
    for call in (lambda: wht.wht_attention_paged4(q, p, p, s, s, i, i[0]), lambda: wht.wht_attention_append4(q, q, q, p, p, s, s, i, i[0], None),
                 lambda: wht.wht_rotary_rotate(q, wht.wht_attention_rope_table(1, 64, device="cpu"))):
        with pytest.raises(RuntimeError, match="needs an AMD GPU"):
            call()


def test_axes():
    assert wht.wht_rotary_axes((2, 1, 3)) == bytes([0, 0, 1, 2, 2, 2])
    assert wht.wht_rotary_axes((2, 1, 3), cyclic=True) == bytes([0, 1, 2, 0, 2, 2])
    assert wht.wht_rotary_axes((3,)) == bytes(3) and wht.wht_rotary_axes((0, 2)) == bytes([1, 1])
    for bad in ((), (1, 2, 3, 4, 5), (1, -1)):
        with pytest.raises(ValueError, match="sections must be"):
            wht.wht_rotary_axes(bad)


def test_short_items_need_no_workspace():
    """They are taken whole, in one launch; more or longer ones leave partial results."""
    need = lambda B, heads, length, prefix=0, D=128: wht.wht_attention4_workspace_bytes(B, B, heads, heads, D, 1, length, prefix, 1)
    assert need(4, 8, 768) == 0 and need(4, 8, 769) > 0 and need(4, 8, 700, 69) > 0
    assert need(32, 8, 2560) == 0 and need(33, 8, 2560) > 0
    assert need(64, 8, 2560, D=64) == 0 and need(65, 8, 100, D=64) > 0


@pytest.mark.parametrize("x,error", [(1 << 31, ValueError), (2.5, ValueError), (None, TypeError), ("x", TypeError)])
def test_numbers_that_do_not_fit_are_refused(x, error):
    with pytest.raises(error, match="max_q must be a whole number"):
        wht.wht_attention4_workspace_bytes(3, 3, 4, 4, 128, x, 128, 0, 1)


@pytest.mark.parametrize("source", ["wht_attention4.hip", "attention4_device.h", "append4_device.h", "rotary_device.h", "attention4_plan.h", "attention_device.h",
                                    *build.ATTENTION4_HEADERS])
def test_an_older_library_is_refused(source, monkeypatch):
    source = os.path.join(build.HERE, "csrc", source)
    real = os.path.getmtime
    build.ensure_built()
    monkeypatch.setattr(os.path, "getmtime", lambda f: real(source) - 1.0 if f == build.ATTENTION4_LIB else max(real(f), real(source)) if f.endswith(".so") else real(f))
    with pytest.raises(RuntimeError, match="older than its source"):
        build.ensure_built()


def test_the_definition_by_hand():
    """A block of 31 ones and a 7: 6 is the largest level, so that the scale is 2, a one 0.5 of it, and the 7 lies halfway between 3 and 4 and goes
    to the even code of 4."""
    x = torch.ones(1, 32, dtype=torch.float64)
    x[0, 31] = -7.0
    codes, scales = check.encode(x)
    assert scales.tolist() == [[128]] and codes.tolist() == [[0x11] * 15 + [0xe1]]
    assert check.decode(codes, scales)[0, 30:].tolist() == [1.0, -8.0]
    # 6 itself keeps the scale 1; the next number above it does not
    assert check.encode(torch.full((1, 32), 6.0, dtype=torch.float64))[1].item() == 127
    assert check.encode(torch.full((1, 32), 6.0 + 2.0 ** -50, dtype=torch.float64))[1].item() == 128
    zero = check.encode(torch.full((1, 32), -0.0, dtype=torch.float64))
    assert zero[0].sum().item() == 0 and zero[1].item() == 3
    assert check.encode(torch.tensor([[float("nan")] + [1.0] * 31], dtype=torch.float64))[1].item() == 255
    e0 = torch.zeros(1, 32, dtype=torch.float64)
    e0[0, 3] = 4.0
    h = check.transform(e0, 4)                                       # one large element becomes 32 of the same size
    assert torch.equal(h.abs(), torch.ones_like(h)) and torch.equal(check.transform(h, 8), e0)


def test_axes_are_taken_number_by_number():
    """bytes() of an array is its memory, of a number so many zeros."""
    want = bytes([0, 1, 2, 1, 0, 2, 2, 1])
    for kind in (bytes, bytearray, list, tuple, iter, memoryview, lambda a: np.array(list(a)), lambda a: np.array(list(a), dtype=np.int16),
                 lambda a: np.array(list(a), dtype=np.uint8)[::1], lambda a: torch.tensor(list(a)), lambda a: torch.tensor(list(a), dtype=torch.int8)):
        assert rotary._axes(kind(want), 16, 3) == want
    assert rotary._axes(None, 16, 3) is None
    for bad in (8, True, "01210221", [0.0] * 8, [300] * 8, [-1] * 8, np.zeros(8), torch.zeros(8), [None] * 8):
        with pytest.raises(TypeError, match="axes must be the axis of each pair"):
            rotary._axes(bad, 16, 3)
    for bad in (np.zeros(4, np.int16), np.zeros(2, np.int32), [0] * 7):
        with pytest.raises(ValueError, match="one number for each of the 8 pairs"):
            rotary._axes(bad, 16, 3)
    with pytest.raises(ValueError, match="below 2"):
        rotary._axes(np.array(list(want)), 16, 2)


def test_selftest_under_sanitizers(tmp_path):
    exe = str(tmp_path / "attention4_san")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", *SAN, "-o", exe, os.path.join(CSRC, "attention4_selftest.cpp")], check=True)
    assert "attention4_selftest: ok" in _run(exe)


@pytest.mark.parametrize("source", ["attention4_plan.h", *build.ATTENTION4_HEADERS])
def test_older_rules_are_refused(source, monkeypatch):
    source = os.path.join(build.HERE, "csrc", source)
    real = os.path.getmtime
    build.ensure_built()
    monkeypatch.setattr(os.path, "getmtime", lambda f: real(source) - 1.0 if f == build.ATTENTION_QUERY_LIB else max(real(f), real(source)) if f.endswith(".so") else real(f))
    with pytest.raises(RuntimeError, match="attention_query.so is older than its source"):
        build.ensure_built()
