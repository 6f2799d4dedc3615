"""LDS places of the 4-bit product kernels are never loaded while they may still be read: the check of
test_lds_schedule_cpu.py, which runs the kernels' source on the host, on the 4-bit kernels."""
import os
import subprocess

import pytest

from test_lds_schedule_cpu import CLANG, CSRC, MAIN, RUNTIME, _counts, needs_clang

RUNTIME4 = RUNTIME + r"""
#define __builtin_amdgcn_raw_buffer_load_b32 trace::load_b8
#define __builtin_amdgcn_s_sleep(x)
struct Two { uint32_t v[2]; uint32_t operator[](int i) const { return v[i]; } };
#define __builtin_amdgcn_permlane16_swap(a, b, ...) (Two{{a, b}})
#define __builtin_amdgcn_update_dpp(a, b, ...) (b)
namespace trace {
// eight records of a lane are a 16-byte store
inline void store() { for (int i = 0; i < 8; ++i) add(ROUND, 0, 1); }
}
"""
# stores are counted where they are made, not by their roundings
rounding = "if (std::is_same<S, __bf16>::value) add(ROUND, 0, 1);"
assert rounding in RUNTIME4
RUNTIME4 = RUNTIME4.replace(rounding, "")
MAIN4 = MAIN
for was, now in (("Fp8Problem", "Fp4Problem"),
                 ("  const int kb = fp8_k_blocks(K);\n", ""),
                 ("  p.kb = kb;\n  p.pitch = fp8_scale_pitch(K);\n",
                  "  p.pitch = fp4_pitch(K);\n  p.kt = p.pitch / 128;\n  p.spitch = fp4_scale_pitch(K);\n")):
    assert was in MAIN4
    MAIN4 = MAIN4.replace(was, now)


def _run(tmp_path, cases, edit=lambda s: s):
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(RUNTIME4)
    source = edit(open(os.path.join(CSRC, "gemm_fp4.hip")).read())
    for store in ("((F32x4*)(y + i * 4))->v =", "((Bf16x8*)(y + i * 2))->v =", "__builtin_nontemporal_store(w, &((Bf16x8*)y)->v);"):
        assert source.count(store) == 1
        source = source.replace(store, "trace::store(), " + store)
    source = source.replace('#include "device_common.h"', f'#include "{CSRC}/device_common.h"')
    (tmp_path / "kernels.h").write_text(source)
    src, exe = tmp_path / "run.cpp", tmp_path / "run"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "hip/hip_runtime.h"\n'
                   + MAIN4.replace("SOURCE", str(tmp_path / "kernels.h")).replace("CASES", cases))
    r = subprocess.run([CLANG, "-O1", "-std=c++17", "-w", "-I", str(tmp_path), str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout.splitlines()


# 24 tiles, of which the block takes three (two of them whole with M = 6100, so that its waits count stores; fp32 rows are
# either all whole or all ragged, as the lanes' records have to agree); K of 3 to 8 tiles
CASES_256 = "\n".join(f'run("256x256", fp4_256_kernel<false>, 4, 1, 6100, {n}, {k}, 2, 2 * 65536 + 2 * 8192);'
                      for k, n in ((600, 256), (1024, 256), (1100, 250), (1500, 256), (1700, 256), (2048, 256)))
CASES_256 += "\n" + "\n".join(f'run("256x256 fp32", fp4_256_kernel<true>, 4, 1, 6144, {n}, {k}, 4, 2 * 65536 + 2 * 8192);'
                              for k, n in ((600, 256), (1024, 256), (2000, 256)))


@needs_clang
def test_places_of_the_256x256_kernel_are_read_before_they_are_loaded_again(tmp_path):
    lines = _run(tmp_path, CASES_256)
    assert len(lines) == 9
    for line in lines:
        c = _counts(line)
        assert c["loads"] > 500 and c["barriers"] > 45 and c["pairs"] > 10000, line
        assert c["races"] == 0 and c["unloaded"] == 0, line


SMALL = [("64x64", "fp4_ring_kernel<{f}, 64, 64, 2, 2, 2, {st}>", 8, 4, 128, 128, (2, 4)),
         ("128x128", "fp4_ring_kernel<{f}, 128, 128, 2, 4, 1, {st}>", 8, 2, 256, 128, (2, 4)),
         ("16x32", "fp4_split_kernel<{f}, 1, 2, 4>", 4, 2, 32, 32, (0,)),
         ("32x32", "fp4_split_kernel<{f}, 2, 2, 4>", 4, 2, 64, 32, (0,))]
CASES_SMALL = "\n".join(f'run("{cfg}", ({form.format(f=f, st=st)}), {waves}, {blocks}, {M}, {N}, {K}, {4 if f == "true" else 2});'
                        for cfg, form, waves, blocks, M, N, stages in SMALL for f in ("false", "true") for st in stages
                        for K in (100, 1280, 3400))


@needs_clang
def test_places_of_the_smaller_tiles_are_read_before_they_are_loaded_again(tmp_path):
    lines = _run(tmp_path, CASES_SMALL)
    assert len(lines) == 36
    for line in lines:
        c = _counts(line)
        assert c["loads"] > 0 and c["pairs"] > 0 and c["races"] == 0 and c["unloaded"] == 0, line


@needs_clang
@pytest.mark.parametrize("was,now", [
    ("wait_vmcnt<24>();  //", "wait_vmcnt<28>();  //"),                                       # ahead of the loop
    ("else wait_vmcnt<24>();", "else wait_vmcnt<28>();"),                                     # in a phase
    ("24 + n * NS < 62 ? 24 + n * NS : 62", "36 + n * NS < 62 ? 36 + n * NS : 62"),           # beside the stores
    ("__builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)\n    if constexpr (st == 1", "if constexpr (st == 1"),  # for reads
    ("using CW = std::integral_constant<int, (c + Q - 1) % Q>;", "using CW = std::integral_constant<int, c>;"),
    ("else if constexpr (i == 9 && st == 1 && c == 3)", "else if constexpr (i == 9 && st == 1 && c == 1)"),
])
def test_the_check_sees_what_comes_too_early(tmp_path, was, now):
    def edit(s):
        assert s.count(was) == 1, was
        return s.replace(was, now)
    lines = _run(tmp_path, CASES_256, edit)
    assert any(_counts(line)["races"] > 0 for line in lines), lines
