"""Host-side checks of the operators around a small cache that need no GPU: parameter blocks, refusals before anything is enqueued,
workspace sizes, and what the compiler made of the kernels."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2605_15508_amd as sts
from paper_2605_15508_amd import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAR = 1 << 40            # an address that nothing looks at
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sts.library_path()):
        build.build(force=True)
    return sts.load_library()


def cache(d=128, **kw):
    base = dict(codes=FAR, scales=FAR, code_stride_b=8 * 4096 * d, code_stride_h=4096 * d, code_stride_n=d, scale_stride_b=8 * 4096 * d // 16,
                scale_stride_h=4096 * d // 16, scale_stride_n=d // 16, N=4096)
    base.update(kw)
    return binding.PackedCache(**base)


def rows(c=None, **kw):
    base = dict(B=1, T=5, Hkv=8, d=128, k=FAR, v=FAR)
    base.update(kw)
    return binding.PackedRowsParams(**base, cache=c if c is not None else cache(base["d"]))


def attn(c=None, **kw):
    base = dict(B=1, Tq=5, Hq=32, Hkv=8, d=128, q=FAR, scale=0.1, out=FAR)
    base.update(kw)
    return binding.PackedAttnParams(**base, cache=c if c is not None else cache(base["d"]))


def window(**kw):
    base = dict(B=1, Tq=5, Hq=32, Hkv=8, d=128, N=4096, q=FAR, k=FAR, v=FAR, kv_stride_b=8 * 4096 * 128, kv_stride_h=4096 * 128, kv_stride_n=128,
                window=512, sinks=4, scale=0.1, out=FAR)
    base.update(kw)
    return binding.WindowParams(**base)


def test_ctypes_structs_match_the_header(tmp_path):
    structs = {"sts_packed_cache": binding.PackedCache, "sts_packed_rows_params": binding.PackedRowsParams,
               "sts_packed_attn_params": binding.PackedAttnParams, "sts_window_params": binding.WindowParams}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sts.h"', "int main(void) {"]
    for cname, cls in structs.items():
        lines.append(f'  printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'  printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sts.h")).read(), flags=re.S)
    for cname, cls in structs.items():
        assert int(got[cname]) == ctypes.sizeof(cls), cname
        for f, _ in cls._fields_:
            assert int(got[f"{cname}.{f}"]) == getattr(cls, f).offset, f"{cname}.{f}"
        body = re.search(r"typedef struct \{([^}]*)\} " + cname + ";", text).group(1)
        assert sorted(re.findall(r"\b\*?([A-Za-z_][A-Za-z0-9_]*)\s*(?:,|;)", body)) == sorted(f for f, _ in cls._fields_), cname


BAD_CACHES = [(dict(N=-1), EINVAL), (dict(page_size=3), EUNSUPPORTED), (dict(page_size=64), EUNSUPPORTED), (dict(code_stride_n=120), EUNSUPPORTED),
              (dict(code_stride_n=64), EUNSUPPORTED), (dict(scale_stride_n=4), EUNSUPPORTED), (dict(scale_stride_n=12), EUNSUPPORTED),
              (dict(code_stride_h=8), EUNSUPPORTED), (dict(code_stride_b=-128), EUNSUPPORTED), (dict(scale_stride_h=-8), EUNSUPPORTED),
              (dict(codes=FAR + 8), EUNSUPPORTED), (dict(scales=FAR + 4), EUNSUPPORTED), (dict(code_stride_n=1 << 27), EUNSUPPORTED),
              (dict(N=0x7fffffff), EUNSUPPORTED), (dict(block_table=FAR, page_size=16, num_pages=0), EINVAL),
              (dict(block_table=FAR, page_size=16, num_pages=4, table_stride=256, code_stride_page=0, scale_stride_page=8), EINVAL),
              (dict(block_table=FAR, page_size=16, num_pages=4, table_stride=255, code_stride_page=128, scale_stride_page=8), EINVAL),
              (dict(block_table=FAR, page_size=16, num_pages=4, table_stride=256, code_stride_page=24, scale_stride_page=8), EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(lib, change, status):
    for f in (lib.sts_packed_store, lib.sts_packed_load):
        assert f(ctypes.byref(rows(cache(**change))), None) == status
    p = attn(cache(**change))
    assert lib.sts_packed_attn(ctypes.byref(p), None) == status
    assert lib.sts_packed_attn_workspace_bytes(ctypes.byref(p)) == 0


@pytest.mark.parametrize("change,status", [(dict(B=-1), EINVAL), (dict(T=-1), EINVAL), (dict(Hkv=0), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
                                           (dict(k=FAR + 8), EUNSUPPORTED), (dict(v=FAR + 2), EUNSUPPORTED), (dict(B=65536), EUNSUPPORTED),
                                           (dict(T=1 << 30, Hkv=8), EUNSUPPORTED), (dict(T=1 << 25, Hkv=8), EUNSUPPORTED)])
def test_rows_that_are_refused(lib, change, status):
    for f in (lib.sts_packed_store, lib.sts_packed_load):
        assert f(ctypes.byref(rows(**change)), None) == status


def test_row_calls_without_rows_and_data(lib):
    for f in (lib.sts_packed_store, lib.sts_packed_load):
        assert f(None, None) == EINVAL
        assert f(ctypes.byref(rows(B=0)), None) == 0 and f(ctypes.byref(rows(T=0)), None) == 0
        assert f(ctypes.byref(rows(cache(codes=None))), None) == EINVAL and f(ctypes.byref(rows(cache(scales=None))), None) == EINVAL
        assert f(ctypes.byref(rows(cache(96), d=96)), None) == EUNSUPPORTED
    assert lib.sts_packed_store(ctypes.byref(rows(cache(N=0, codes=None, scales=None))), None) == 0       # no place for any row


HEADS = [(dict(B=-1), EINVAL), (dict(Tq=0), EINVAL), (dict(Hq=30), EINVAL), (dict(Hkv=0), EINVAL), (dict(Hq=512, Hkv=256), EUNSUPPORTED),
         (dict(Hq=32, Hkv=1), EUNSUPPORTED), (dict(out_dtype=2), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=-3e38), EINVAL),
         (dict(k_new=FAR), EINVAL), (dict(v_new=FAR), EINVAL), (dict(k_new=FAR + 8, v_new=FAR), EUNSUPPORTED), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
         (dict(q=FAR + 8), EUNSUPPORTED), (dict(out=FAR + 4), EUNSUPPORTED), (dict(), EWORKSPACE), (dict(workspace=FAR, workspace_bytes=100), EWORKSPACE),
         (dict(workspace=FAR + 128, workspace_bytes=1 << 30), EWORKSPACE)]


@pytest.mark.parametrize("change,status", HEADS + [(dict(Tq=17), EUNSUPPORTED), (dict(counts=FAR), EINVAL), (dict(kmax=4), EINVAL), (dict(indices=FAR, kmax=-1), EINVAL),
                                                   (dict(indices=FAR, kmax=4, seq_lens=FAR), EINVAL), (dict(indices=FAR, kmax=0x7fffffff), EUNSUPPORTED),
                                                   (dict(indices=FAR, kmax=4, idx_stride_b=100), EINVAL), (dict(indices=FAR, kmax=4, idx_stride_b=-128), EINVAL),
                                                   (dict(indices=FAR, kmax=4, cnt_stride_b=31), EINVAL)])
def test_packed_attention_that_is_refused(lib, change, status):
    assert lib.sts_packed_attn(ctypes.byref(attn(**change)), None) == status


def test_packed_attention_without_a_batch_or_a_map(lib):
    assert lib.sts_packed_attn(None, None) == EINVAL and lib.sts_packed_attn_workspace_bytes(None) == 0
    assert lib.sts_packed_attn(ctypes.byref(attn(B=0)), None) == 0
    bad = (ctypes.c_int32 * 32)(*[-1] * 32)
    p = attn(indices=FAR, kmax=4, head_map=ctypes.cast(bad, ctypes.c_void_p))
    assert lib.sts_packed_attn(ctypes.byref(p), None) == EINVAL
    p = attn(head_map=ctypes.cast(bad, ctypes.c_void_p))
    assert lib.sts_packed_attn(ctypes.byref(p), None) == EINVAL            # a map without lists
    p = attn(cache(N=0), indices=FAR, kmax=4)
    assert lib.sts_packed_attn(ctypes.byref(p), None) == EINVAL            # lists into a cache without tokens


@pytest.mark.parametrize("change,status", HEADS + [(dict(N=-1), EINVAL), (dict(window=0), EINVAL), (dict(window=-5), EINVAL), (dict(sinks=-1), EINVAL),
                                                   (dict(d=96), EUNSUPPORTED), (dict(N=0x7fffffff), EUNSUPPORTED), (dict(k_new=FAR, v_new=FAR, Tq=17), EUNSUPPORTED),
                                                   (dict(k_new=FAR, v_new=FAR, window=4), EUNSUPPORTED), (dict(kv_stride_n=64), EUNSUPPORTED),
                                                   (dict(kv_stride_n=132), EUNSUPPORTED), (dict(kv_stride_h=4), EUNSUPPORTED), (dict(kv_stride_b=-128), EUNSUPPORTED),
                                                   (dict(kv_stride_n=1 << 26), EUNSUPPORTED), (dict(page_size=5), EUNSUPPORTED), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
                                                   (dict(k=FAR + 8), EUNSUPPORTED), (dict(block_table=FAR, page_size=16, num_pages=0, kv_stride_page=128), EINVAL),
                                                   (dict(block_table=FAR, page_size=16, num_pages=9, kv_stride_page=0), EINVAL),
                                                   (dict(block_table=FAR, page_size=16, num_pages=9, kv_stride_page=132, table_stride=256), EUNSUPPORTED),
                                                   (dict(block_table=FAR, page_size=16, num_pages=9, kv_stride_page=128, table_stride=255), EINVAL),
                                                   (dict(Tq=1 << 30, Hq=64, Hkv=8), EUNSUPPORTED), (dict(Tq=4096, B=1 << 17), EUNSUPPORTED), (dict(Tq=64, workspace=FAR, workspace_bytes=64), EWORKSPACE)])
def test_window_attention_that_is_refused(lib, change, status):
    assert lib.sts_window_attn(ctypes.byref(window(**change)), None) == status


def test_window_attention_without_a_batch(lib):
    assert lib.sts_window_attn(None, None) == EINVAL and lib.sts_window_attn_workspace_bytes(None) == 0
    assert lib.sts_window_attn(ctypes.byref(window(B=0)), None) == 0


def test_workspaces_go_by_the_shape_alone(lib):
    size = lambda p: lib.sts_packed_attn_workspace_bytes(ctypes.byref(p))  # noqa: E731
    assert size(attn()) == size(attn(q=None, out=None, scale=3.0)) > 256
    assert size(attn(cache(N=64))) >= 256
    w = lambda **kw: lib.sts_window_attn_workspace_bytes(ctypes.byref(window(**kw)))  # noqa: E731
    assert w() == w(q=None, k=None) > 256
    assert w(Tq=100000, N=100000) == 256               # a block for every compute unit and more: nothing to put together
    assert w(Tq=64) > 256
    # a window asks for no more than its keys take, however long the cache
    assert w(N=1 << 20, window=100) <= w(N=1 << 20, window=4096)


def test_enums_and_kinds():
    text = open(os.path.join(ROOT, "include", "sts.h")).read()
    for name, value in binding.KERNEL_KINDS.items():
        if value >= 17:
            assert re.search(rf"STS_K_{name.upper()} = {value},", text), name


@pytest.fixture(scope="module")
def resources():
    if not os.path.exists(build.RESOURCES) or build.needs_build():
        build.build(force=True)
    return build.kernel_resources()


@pytest.mark.parametrize("name,forms,most", [("packed_store_kernel", 2, 64), ("packed_load_kernel", 2, 64), ("window_prompt_kernel", 6, 256),
                                             ("window_combine_kernel", 2, 64), ("cache_attn_kernel", 20, 256)])
def test_kernels_fit_their_registers(resources, name, forms, most):
    found = {k: v for k, v in resources.items() if f"{len(name)}{name}I" in k}
    assert len(found) == forms
    for k, v in found.items():
        assert v["ScratchSize"] == 0 and v["VGPRs"] <= most, k
        assert v["AGPRs"] == 0, k
        assert v["LDS Size"] <= 80 * 1024, k                     # two workgroups per compute unit


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    out = tmp_path_factory.mktemp("listing") / "attn_cache.s"
    subprocess.run([build._hipcc(), *[f for f in build.COMMON if not f.startswith("-Rpass") and f != "-fPIC"], "-S", "--cuda-device-only", os.path.join(build.CSRC, "attn_cache.hip"),
                    "-o", str(out)], check=True, capture_output=True)
    return out.read_text()


def test_scaled_products_do_not_write_to_their_operands(listing):
    """The instruction takes eight passes; its result may be the third operand's registers or none of any operand's, which the compiler does
    not see to by itself."""
    def regs(s):
        m = re.match(r"[va]\[(\d+):(\d+)\]$", s)
        if m:
            return {s[0] + str(i) for i in range(int(m.group(1)), int(m.group(2)) + 1)}
        return {s} if re.match(r"[va]\d+$", s) else set()

    seen = 0
    for ln in listing.splitlines():
        m = re.match(r"\s+v_mfma_scale_f32_16x16x128_f8f6f4 (\S+), (\S+), (\S+), (\S+), (\S+), (\S+) ", ln + " ")
        if not m:
            continue
        d, a, b, c, sa, sb = (regs(x) for x in m.groups())
        seen += 1
        assert d and not d & (a | b | sa | sb), ln
        assert not c or c == d or not c & d, ln
    assert seen >= 100


def test_lds_arrays_are_accessed_as_one_type(tmp_path):
    from test_lds_types import access_types

    out = tmp_path / "x.ll"
    subprocess.run([build._hipcc(), "--offload-arch=gfx950", "--cuda-device-only", "-std=c++17", "-O3", "-w", "-Xclang", "-disable-llvm-passes",
                    "-S", "-emit-llvm", "-o", str(out), os.path.join(build.CSRC, "attn_cache.hip")], check=True)
    types = access_types(out.read_text())
    assert any("lds_sc" in k for k in types)
    bad = {k: v for k, v in types.items() if len(set(v) - {"omnipotent char"}) > 1}
    assert not bad, bad
