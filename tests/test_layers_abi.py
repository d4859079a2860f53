"""Host-side checks of the layers over packed batches that need no GPU: parameter blocks, refusals before anything is enqueued, workspace
sizes, what the compiler made of the kernels."""
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


def prompt(**kw):
    base = dict(B=2, T=500, Hq=32, Hkv=8, d=128, q=FAR, k=FAR, v=FAR, q_stride_n=4096, q_stride_h=128, kv_stride_n=1024, kv_stride_h=128, starts=FAR,
                scale=0.1, out=FAR)
    base.update(kw)
    return binding.PromptParams(**base)


def linear(**kw):
    base = dict(B=2, T=5000, Hq=32, Hkv=8, d=128, q=FAR, k=FAR, v=FAR, q_stride_n=4096, q_stride_h=128, kv_stride_n=1024, kv_stride_h=128, decay=FAR,
                starts=FAR, scale=0.1, state=FAR, state_stride=8 * 128 * 128, num_slots=2, state_out=FAR, state_out_stride=8 * 128 * 128, num_slots_out=2,
                out=FAR, workspace=FAR, workspace_bytes=1 << 34)
    base.update(kw)
    return binding.LinearParams(**base)


def test_ctypes_structs_match_the_header(tmp_path):
    structs = {"sts_prompt_params": binding.PromptParams, "sts_linear_params": binding.LinearParams}
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


BOTH = [(dict(B=-1), EINVAL), (dict(T=-1), EINVAL), (dict(Hq=30), EINVAL), (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(d=96), EUNSUPPORTED),
        (dict(Hq=512, Hkv=256), EUNSUPPORTED), (dict(Hq=32, Hkv=1), EUNSUPPORTED), (dict(out_dtype=2), EINVAL), (dict(scale=float("nan")), EINVAL),
        (dict(scale=-3e38), EINVAL), (dict(kv_stride_n=120), EUNSUPPORTED), (dict(kv_stride_n=1028), EUNSUPPORTED), (dict(kv_stride_n=-1024), EUNSUPPORTED),
        (dict(kv_stride_h=4), EUNSUPPORTED), (dict(kv_stride_h=-128), EUNSUPPORTED), (dict(kv_stride_n=1 << 26), EUNSUPPORTED), (dict(kv_stride_n=(1 << 24) + 8), EUNSUPPORTED), (dict(q_stride_n=1 << 25), EUNSUPPORTED), (dict(q_stride_n=64), EUNSUPPORTED),
        (dict(q_stride_n=4100), EUNSUPPORTED), (dict(q_stride_h=-8), EUNSUPPORTED), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(k=None), EINVAL),
        (dict(v=None), EINVAL), (dict(q=FAR + 8), EUNSUPPORTED), (dict(k=FAR + 2), EUNSUPPORTED), (dict(v=FAR + 8), EUNSUPPORTED), (dict(out=FAR + 4), EUNSUPPORTED),
        (dict(T=1 << 30), EUNSUPPORTED), (dict(B=0x7fffffff), EUNSUPPORTED), (dict(B=1 << 24, Hkv=32), EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BOTH + [(dict(starts=None), EINVAL)])
def test_prompts_that_are_refused(lib, change, status):
    assert lib.sts_prompt_attn(ctypes.byref(prompt(**change)), None) == status


@pytest.mark.parametrize("change,status", BOTH + [
    (dict(max_len=-1), EINVAL), (dict(starts=None, B=3), EINVAL), (dict(decay=None), EINVAL), (dict(num_slots=1), EINVAL), (dict(num_slots_out=1), EINVAL), (dict(num_slots=-1, slots=FAR), EINVAL),
    (dict(state=None, slots=FAR), EINVAL), (dict(state_out=None, slots_out=FAR), EINVAL), (dict(state_stride=8 * 128 * 128 - 4), EUNSUPPORTED),
    (dict(state_out_stride=0), EUNSUPPORTED), (dict(state_stride=8 * 128 * 128 + 2), EUNSUPPORTED), (dict(state=FAR + 4), EUNSUPPORTED), (dict(state_out=FAR + 8), EUNSUPPORTED),
    (dict(workspace=None), EWORKSPACE), (dict(workspace_bytes=1000), EWORKSPACE), (dict(workspace=FAR + 128), EWORKSPACE)])
def test_linear_attention_that_is_refused(lib, change, status):
    assert lib.sts_linear_attn(ctypes.byref(linear(**change)), None) == status


def test_calls_without_anything_to_do(lib):
    assert lib.sts_prompt_attn(None, None) == EINVAL and lib.sts_linear_attn(None, None) == EINVAL and lib.sts_linear_attn_workspace_bytes(None) == 0
    none = dict(q=None, k=None, v=None, out=None, starts=None)
    assert lib.sts_prompt_attn(ctypes.byref(prompt(B=0, **none)), None) == 0 and lib.sts_prompt_attn(ctypes.byref(prompt(T=0, **none)), None) == 0
    assert lib.sts_linear_attn(ctypes.byref(linear(B=0, workspace=None)), None) == 0
    assert lib.sts_linear_attn(ctypes.byref(linear(q=None, out=None, state_out=None, num_slots_out=0, workspace=None)), None) == 0


def test_workspaces_go_by_the_shape_alone(lib):
    size = lambda **kw: lib.sts_linear_attn_workspace_bytes(ctypes.byref(linear(**kw)))  # noqa: E731
    assert size() == size(q=None, out=None, k=None, state=None, scale=2.0) > 8 * 128 * 128 * 4
    assert size(max_len=16) == 256                     # row by row
    assert size(max_len=100, Hkv=32) == 256            # no sequence is cut, no group shares a state
    assert size(starts=None, B=5000) == 256 and size(starts=None, B=5) > 256 and size(starts=None, B=50, Hkv=32) == 256
    assert size(max_len=5000) == size(max_len=0) == size(max_len=9000)
    assert size(d=96) == 0


@pytest.fixture(scope="module")
def resources():
    if not os.path.exists(build.RESOURCES) or build.needs_build():
        build.build(force=True)
    return build.kernel_resources()


@pytest.mark.parametrize("name,forms", [("prompt_attn_kernel", 2), ("linear_step_kernel", 6), ("linear_chunk_kernel", 6), ("linear_carry_kernel", 2)])
def test_kernels_fit_their_registers(resources, name, forms):
    found = {k: v for k, v in resources.items() if f"{len(name)}{name}I" in k}
    assert len(found) == forms
    for k, v in found.items():
        assert v["ScratchSize"] == 0 and v["AGPRs"] == 0, k
        # two workgroups of four waves on a compute unit, three of the small prompts', four of two waves of the small chunks'; three or more of the steps'
        half = "ILi64E" in k
        most = {"prompt_attn_kernel": 168 if half else 256, "linear_step_kernel": 168, "linear_chunk_kernel": 256, "linear_carry_kernel": 128}[name]
        lds = {"prompt_attn_kernel": 160 // 3 if half else 80, "linear_step_kernel": 160 // 5, "linear_chunk_kernel": 40 if half else 80, "linear_carry_kernel": 0}[name]
        assert v["VGPRs"] <= most and v["LDS Size"] <= lds * 1024, k


def test_enums_and_kinds():
    text = open(os.path.join(ROOT, "include", "sts.h")).read()
    for name, value in binding.KERNEL_KINDS.items():
        if value >= 21:
            assert re.search(rf"STS_K_{name.upper()} = {value},", text), name
    assert f"STS_K_COUNT_ = {max(binding.KERNEL_KINDS.values()) + 1}" in text
