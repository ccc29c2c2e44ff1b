"""What the binding of the 4-bit paged cache passes on to the library and what it
refuses, and the C ABI's refusals and structs, without a GPU."""

import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from paper_2607_08565_gb300 import build_lib
from test_kv_refusals import Library, on, plan

BF, E4M3, U8 = torch.bfloat16, torch.float8_e4m3fn, torch.uint8
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODES, SCALES = (3, 16, 2, 32), (3, 16, 2, 4)


@pytest.fixture
def kv(monkeypatch):
    lib = Library()
    monkeypatch.setattr(pkg, "lib", lambda: lib)
    monkeypatch.setattr(pkg, "smetric_kv_create", lambda cfg: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    kv = pkg.SMetricKV4(head_dim=64, num_q_heads=4, num_kv_heads=2, page_size=16, num_pages=3, max_batch_requests=2, max_batch_tokens=8)
    kv.library = lib
    kv.plan(*(on(x, 0) for x in plan()), 4)
    lib.calls.clear()
    yield kv
    kv.handle = None


def cache(exp=0):
    return pkg.Cache4(on(torch.zeros(CODES, dtype=U8), 0), on(torch.zeros(SCALES, dtype=E4M3), 0), exp)


def heads(n=4, h=2):
    return on(torch.zeros(n, h, 64, dtype=BF), 0)


def read_args():
    return dict(offsets=on(torch.tensor([0, 4]), 0), pages=on(torch.zeros(1, 2, dtype=torch.int32), 0), n_rows=4,
                first=on(torch.zeros(1, dtype=torch.int32), 0), k_out=heads(), v_out=heads())


def call(kv, name, k_cache, v_cache):
    if name == "append":
        return kv.append(k_cache, v_cache, heads(), heads(), q=heads(h=4), q_out=heads(h=4))
    if name == "paged_attention":
        return kv.paged_attention(heads(h=4), k_cache, v_cache, out=heads(h=4))
    return kv.read(k_cache, v_cache, **read_args())


CALLS = {"append": "smetric_kvq_append", "paged_attention": "smetric_kvq_attention", "read": "smetric_kvq_read"}


@pytest.mark.parametrize("name", CALLS)
def test_caches_come_through(kv, name):
    wide = on(torch.zeros(3, 2, 20, 48, dtype=U8), 0)  # heads outside tokens, room between rows
    codes = wide[:, :, 2:18, 16:].transpose(1, 2)
    codes.at = 0
    k_cache, v_cache = pkg.Cache4(codes, cache().scales, -7), cache(5)
    call(kv, name, k_cache, v_cache)
    assert kv.library.calls == [CALLS[name]]
    k, v = kv.library.args[1:3]
    assert (k.d_codes, k.page_stride, k.token_stride, k.head_stride, k.exp) == (codes.data_ptr(), 2 * 20 * 48, 48, 20 * 48, -7)
    assert (v.page_stride, v.token_stride, v.head_stride, v.exp, v.reserved) == (16 * 64, 64, 32, 5, 0)
    assert (v.d_scales, v.scale_page_stride, v.scale_token_stride, v.scale_head_stride) == (v_cache.scales.data_ptr(), 16 * 8, 8, 4)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("field,value", [
    ("codes", torch.zeros(CODES, dtype=torch.int8)), ("codes", torch.zeros(3, 16, 2, 64, dtype=U8)), ("codes", torch.zeros(2, 16, 2, 32, dtype=U8)),
    ("codes", torch.zeros(3, 16, 2, 64, dtype=U8)[..., ::2]), ("scales", torch.zeros(SCALES, dtype=U8)),
    ("scales", torch.zeros(3, 16, 2, 8, dtype=U8).view(E4M3)), ("scales", torch.zeros(3, 16, 2, 8, dtype=U8)[..., ::2].view(E4M3)),
    ("exp", 65), ("exp", -65), ("exp", 2 ** 32),
])
def test_bad_caches_are_refused(kv, name, which, field, value):
    caches = [cache(), cache()]
    caches[which] = caches[which]._replace(**{field: on(value, 0) if isinstance(value, torch.Tensor) else value})
    with pytest.raises(ValueError):
        call(kv, name, *caches)
    assert not kv.library.calls


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("device", [-1, 1])  # the host, another GPU
@pytest.mark.parametrize("field", ["codes", "scales"])
def test_caches_elsewhere_are_refused(kv, name, device, field):
    for which in range(2):
        caches = [cache(), cache()]
        getattr(caches[which], field).at = device
        with pytest.raises(ValueError, match="device|cuda"):
            call(kv, name, *caches)
    assert not kv.library.calls


@pytest.mark.parametrize("name", CALLS)
def test_caches_of_16_bits_are_refused(kv, name):
    with pytest.raises(ValueError, match="Cache4"):
        call(kv, name, torch.zeros(3, 16, 2, 64, dtype=BF), cache())
    assert not kv.library.calls


@pytest.mark.parametrize("name", ["offsets", "pages", "first", "k_out", "v_out"])
@pytest.mark.parametrize("device", [-1, 1])
def test_reads_elsewhere_are_refused(kv, name, device):
    args = read_args()
    args[name].at = device
    with pytest.raises(ValueError, match="device|cuda"):
        kv.read(cache(), cache(), **args)
    assert not kv.library.calls


@pytest.mark.parametrize("name,value", [
    ("offsets", torch.tensor([0, 4], dtype=torch.int32)), ("offsets", torch.zeros(0, dtype=torch.int64)), ("offsets", torch.tensor([[0, 4]])),
    ("offsets", torch.tensor([0, 1, 4])), ("offsets", torch.tensor([0, 1, 4, 4])[::2]), ("pages", torch.zeros(1, 2)),
    ("pages", torch.zeros(2, dtype=torch.int32)), ("pages", torch.zeros(2, 2, dtype=torch.int32)), ("pages", torch.zeros(1, 4, dtype=torch.int32)[:, ::2]),
    ("first", torch.zeros(1)), ("first", torch.zeros(2, dtype=torch.int32)), ("k_out", torch.zeros(3, 2, 64, dtype=BF)),
    ("v_out", torch.zeros(4, 2, 64)), ("k_out", torch.zeros(4, 64, 2, dtype=BF).transpose(1, 2)),
])
def test_bad_reads_are_refused(kv, name, value):
    with pytest.raises(ValueError):
        kv.read(cache(), cache(), **{**read_args(), name: on(value, 0)})
    assert not kv.library.calls


def test_reads_without_a_first_and_of_one_cache(kv):
    args = read_args()
    args["first"] = None
    assert kv.read(cache(), None, **args) == (args["k_out"], None)
    handle, k, v, offsets, n, n_rows, first, pages, most, stride, kh, vh = kv.library.args[:12]
    assert (n, n_rows, first, most, stride) == (1, 4, None, 2, 2) and vh.d_data is None and v.d_codes is None and kh.d_data


@pytest.fixture(scope="module")
def L():
    build_lib.build()
    return C.CDLL(build_lib.LIB)


@pytest.mark.parametrize("bad", [dict(head_dim=16), dict(head_dim=48), dict(head_dim=80), dict(head_dim=112), dict(flags=3), dict(flags=1),
                                 dict(flags=6), dict(page_size=8), dict(num_q_heads=6)])
def test_create_refuses(L, bad):
    cfg = dict(head_dim=64, num_q_heads=8, num_kv_heads=4, page_size=16, dtype=0, flags=pkg.SMETRIC_KV_4BIT, num_pages=4, max_batch_requests=2,
               max_batch_tokens=8)
    cfg.update(bad)
    h = C.c_void_p(1)
    assert L.smetric_kv_create(C.byref(pkg.smetric_kv_config(**cfg)), C.byref(h)) == pkg.SMETRIC_ERR_INVALID_ARG
    assert not h.value


def test_null_handles_are_refused():
    build_lib.build()
    lib = pkg.lib()
    no, t, c = pkg.smetric_heads(), pkg.smetric_kv_transform(), pkg.smetric_kvq_cache()
    bad = pkg.SMETRIC_ERR_INVALID_ARG
    assert lib.smetric_kvq_append(None, c, c, no, no, no, no, t, None) == bad
    assert lib.smetric_kvq_attention(None, c, c, no, 1.0, no, None, None) == bad
    assert lib.smetric_kvq_read(None, c, c, None, 0, 0, None, None, 0, 0, no, no, None) == bad


def test_struct_layout_from_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    t = pkg.smetric_kvq_cache
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "smetric.h"', "int main(void) {",
             '  printf("size %zu\\n", sizeof(smetric_kvq_cache));']
    lines += [f'  printf("{f} %zu\\n", offsetof(smetric_kvq_cache, {f}));' for f, _ in t._fields_]
    src, exe = tmp_path / "layout.c", str(tmp_path / "layout")
    src.write_text("\n".join(lines + ["  return 0;", "}", ""]))
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    seen = dict(x.split() for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines())
    assert C.sizeof(t) == int(seen["size"])
    for f, _ in t._fields_:
        assert getattr(t, f).offset == int(seen[f]), f
