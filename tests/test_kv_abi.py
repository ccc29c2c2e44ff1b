"""The paged KV$ part of the C ABI: refusals that need no GPU, and the structs'
layout against the binding's from plain C."""

import ctypes as C
import os
import shutil
import subprocess

import pytest

import paper_2607_08565_gb300 as pkg
from paper_2607_08565_gb300 import build_lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ("smetric_kv_config", "smetric_heads", "smetric_kv_cache", "smetric_kv_transform")


@pytest.fixture(scope="module")
def L():
    build_lib.build()
    return pkg.lib()


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=8), dict(head_dim=72), dict(head_dim=144), dict(num_kv_heads=0), dict(num_q_heads=6),
    dict(num_q_heads=2), dict(num_q_heads=4 * 129), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(dtype=2),
    dict(dtype=-1), dict(flags=1), dict(num_pages=0), dict(num_pages=1 << 31), dict(max_batch_requests=-1),
    dict(max_batch_requests=(1 << 20) + 1), dict(max_batch_tokens=-1), dict(max_batch_tokens=(1 << 26) + 1),
])
def test_create_refuses(L, bad):
    cfg = dict(head_dim=64, num_q_heads=8, num_kv_heads=4, page_size=16, dtype=0, flags=0, num_pages=4, max_batch_requests=2,
               max_batch_tokens=8)
    cfg.update(bad)
    h = C.c_void_p(1)
    assert L.smetric_kv_create(C.byref(pkg.smetric_kv_config(**cfg)), C.byref(h)) == pkg.SMETRIC_ERR_INVALID_ARG
    assert not h.value


def test_null_handles_are_refused(L):
    no, t, c = pkg.smetric_heads(), pkg.smetric_kv_transform(), pkg.smetric_kv_cache()
    bad = pkg.SMETRIC_ERR_INVALID_ARG
    assert L.smetric_kv_create(None, None) == bad
    assert L.smetric_kv_destroy(None) == pkg.SMETRIC_OK
    assert L.smetric_kv_plan(None, None, 0, 0, None, None, 0, 0, 0, None) == bad
    assert L.smetric_kv_append(None, c, no, no, no, no, t, None) == bad
    assert L.smetric_qk_norm_rope(None, no, no, None, 0, t, no, no, None) == bad
    assert L.smetric_paged_attention(None, c, no, 1.0, no, None, None) == bad
    assert L.smetric_kv_status(None, None) == bad
    assert L.smetric_kv_launch_count(None) == 0


def test_struct_layout_from_c(tmp_path, L):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "smetric.h"', "int main(void) {"]
    for s in STRUCTS:
        lines.append(f'  printf("{s} %zu\\n", sizeof({s}));')
        for f, _ in getattr(pkg, s)._fields_:
            lines.append(f'  printf("{s}.{f} %zu\\n", offsetof({s}, {f}));')
    src, exe = tmp_path / "layout.c", str(tmp_path / "layout")
    src.write_text("\n".join(lines + ["  return 0;", "}", ""]))
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    seen = dict(x.split() for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines())
    for s in STRUCTS:
        t = getattr(pkg, s)
        assert C.sizeof(t) == int(seen[s]), s
        for f, _ in t._fields_:
            assert getattr(t, f).offset == int(seen[f"{s}.{f}"]), f
