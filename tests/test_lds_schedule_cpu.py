"""LDS places of the 8-bit product kernels are never loaded while they may still be read.

Those kernels move their operands by direct-to-LDS loads that the compiler does not
order: the source counts the waits (vmcnt for loads and stores, lgkmcnt for LDS reads)
and places the block barriers by hand.  This test runs the kernels' own source on the
host, lane by lane, with the target's builtins replaced by recorders, and puts the
waves' records together.  For every LDS read and every load into the same 64 bytes it
demands one of

 * the load is before the read: its wave waited for it and then, if that is another
   wave than the reader's, passed a block barrier that the reader passed ahead of the read;
 * the load is after the read: the reader waited for the read's data and then, if the
   loader is another wave, passed a barrier that the loader passed ahead of the load;

and that each place that is read was loaded before (the bias apart, which the first
tile reads for the sums of a tile before it that does not exist).  Between two barriers waves run in
any order, so anything else is a race, however long a load takes.  Only the waits in
the source count; those that the compiler adds ahead of a register's use come later.
"""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_01565_amd", "csrc")
CLANG = next((p for p in ("/opt/rocm/llvm/bin/clang++", shutil.which("clang++")) if p and os.path.exists(p)), None)

# what the sources take from <hip/hip_runtime.h>, with recorders in place of what touches LDS or waits
RUNTIME = r"""
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>
#include <algorithm>
#include <map>
#include <set>
#include <string>
#include <type_traits>
#include <utility>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __forceinline__ inline __attribute__((always_inline))
#define __launch_bounds__(...)
#define __shared__ static __attribute__((aligned(1024)))
#define address_space(n)
#define hipLaunchKernelGGL(...) ((void)0)
typedef int hipError_t;
typedef void* hipStream_t;
enum { hipSuccess = 0 };
inline int hipGetLastError() { return 0; }
struct dim3 { unsigned x, y, z; dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {} };
struct uint2 { uint32_t x, y; };
struct alignas(16) uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
struct alignas(16) float4 { float x, y, z, w; };
inline dim3 blockIdx, gridDim, threadIdx;
using std::max;
using std::min;
inline float __uint_as_float(uint32_t v) { float f; memcpy(&f, &v, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t v; memcpy(&v, &f, 4); return v; }
inline float __expf(float x) { return expf(x); }
inline float __shfl_xor(float x, int, int) { return x; }

namespace trace {
// LOAD: to LDS; OTHER: another vector memory access; READ: of LDS; VM, LGKM: a wait with its count
enum Kind { LOAD, OTHER, READ, VM, LGKM, BARRIER, ROUND };
struct Event { Kind kind; long at; int n; };
struct Lane { std::vector<Event> ev; };
inline Lane* lane;
inline char *lds = nullptr, *lds_end = nullptr;   // of the kernel that runs
inline void add(Kind k, long at, int n) { lane->ev.push_back({k, at, n}); }
inline void statement(const char* s) {
  if (strstr(s, "s_barrier")) add(BARRIER, 0, 0);
}
inline void waitcnt(int v) {
  const int vm = (v & 15) | (v >> 14 & 3) << 4, lgkm = v >> 8 & 15;
  if (vm < 63) add(VM, 0, vm);
  if (lgkm < 15) add(LGKM, 0, lgkm);
}
template <class T, class S>
T cast(const S& s) {
  const char* p = (const char*)&s;
  if (p >= lds && p < lds_end) add(READ, p - lds, (int)sizeof s);
  if (std::is_same<S, __bf16>::value) add(ROUND, 0, 1);   // a bf16 output: eight make a 16-byte store
  T t;
  static_assert(sizeof(T) == sizeof(S), "bit cast");
  memcpy(&t, p, sizeof t);
  return t;
}
struct Buffer { const char* base; int bytes; };
inline Buffer buffer(void* p, short, int n, int) { return {(const char*)p, n}; }
inline void load_lds(Buffer, void* to, int size, int, int, int, int) { add(LOAD, (char*)to - lds, size < 4 ? 4 : size); }
inline int load_b8(Buffer, int, int, int) { add(OTHER, 0, 1); return 127; }
inline void syncthreads() { add(VM, 0, 0); add(LGKM, 0, 0); add(BARRIER, 0, 0); }
}  // namespace trace

// asm volatile("...") -> the statement's text
#define asm
#define volatile(...) trace::statement(#__VA_ARGS__)
#define __syncthreads trace::syncthreads
#define __builtin_bit_cast(T, v) trace::cast<T>(v)
#define __amdgpu_buffer_rsrc_t trace::Buffer
#define __builtin_amdgcn_make_buffer_rsrc trace::buffer
#define __builtin_amdgcn_raw_ptr_buffer_load_lds trace::load_lds
#define __builtin_amdgcn_raw_buffer_load_b8 trace::load_b8
#define __builtin_amdgcn_s_waitcnt trace::waitcnt
#define __builtin_amdgcn_sched_barrier(x)
#define __builtin_amdgcn_readfirstlane(x) (x)
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __any(x) (false)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, ...) (c)
#define __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, ...) (c)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, ...) bf16x2_t{(__bf16)0.f, (__bf16)0.f}
"""

MAIN = r"""
#include "SOURCE"

namespace dit {
namespace {

struct Wave {
  struct Event { trace::Kind kind; std::set<int> places; int n; int barriers; };
  std::vector<Event> ev;
  int barriers = 0;
};

struct Result { long pairs = 0, races = 0, unloaded = 0, loads = 0, barriers = 0; std::string first; };

// Runs block 0 of a grid of one block, of `waves` waves.
template <class Kernel>
std::vector<Wave> record(Kernel kernel, const Fp8Problem& p, int waves, int blocks) {
  std::vector<Wave> out(waves);
  blockIdx = dim3(0, 0, 0);
  gridDim = dim3(blocks);
  for (int w = 0; w < waves; ++w) {
    std::vector<trace::Lane> lanes(64);
    for (int l = 0; l < 64; ++l) {
      trace::lane = &lanes[l];
      threadIdx = dim3(w * 64 + l, 0, 0);
      kernel(p);
    }
    // Put together: the lanes' records agree but for addresses, and for stores, of which a wave makes as many as its
    // lane with the fewest (a wave whose lanes differ makes more, which makes its counted waits stricter).
    std::vector<size_t> at(64, 0);
    std::vector<long> rounds(64, 0);
    for (;;) {
      for (int l = 0; l < 64; ++l)
        for (; at[l] < lanes[l].ev.size() && lanes[l].ev[at[l]].kind == trace::ROUND; ++at[l]) ++rounds[l];
      const long stores = *std::min_element(rounds.begin(), rounds.end()) / 8;
      const bool end = at[0] >= lanes[0].ev.size();
      // stores are issued when their last value is rounded
      for (int i = 0; i < stores; ++i) out[w].ev.push_back({trace::OTHER, {}, 1, out[w].barriers});
      std::fill(rounds.begin(), rounds.end(), 0);
      if (end) break;
      const trace::Event& e0 = lanes[0].ev[at[0]];
      Wave::Event e{e0.kind, {}, e0.n, out[w].barriers};
      for (int l = 0; l < 64; ++l) {
        // lanes that end early (rows that do not exist) take no more part
        if (at[l] >= lanes[l].ev.size()) continue;
        const trace::Event& x = lanes[l].ev[at[l]++];
        if (x.kind != e0.kind || (x.kind != trace::READ && x.n != e0.n)) { printf("lanes differ\n"); exit(2); }
        const long a = x.kind == trace::LOAD ? x.at + l * x.n : x.at;
        if (x.kind == trace::LOAD || x.kind == trace::READ)
          for (long b = a >> 6; b <= (a + x.n - 1) >> 6; ++b) e.places.insert((int)b);
      }
      if (e.kind == trace::BARRIER) ++out[w].barriers;
      out[w].ev.push_back(e);
    }
  }
  return out;
}

// places from byte `free` on may be read before they are loaded
Result check(const std::vector<Wave>& waves, long free) {
  constexpr int NEVER = 1 << 30;
  struct Load { int wave, index, issued, waited_index, waited; };
  Result r;
  std::map<int, std::vector<Load>> loads;
  for (int w = 0; w < (int)waves.size(); ++w) {
    const auto& ev = waves[w].ev;
    std::vector<int> flight;  // vector memory accesses that no wait has covered
    std::map<int, Load> mine;
    for (int i = 0; i < (int)ev.size(); ++i) {
      if (ev[i].kind == trace::LOAD || ev[i].kind == trace::OTHER) {
        flight.push_back(i);
        if (ev[i].kind == trace::LOAD) mine[i] = {w, i, ev[i].barriers, NEVER, NEVER}, ++r.loads;
      } else if (ev[i].kind == trace::VM) {
        while ((int)flight.size() > ev[i].n) {
          const int k = flight.front();
          flight.erase(flight.begin());
          if (mine.count(k)) mine[k].waited_index = i, mine[k].waited = ev[i].barriers;
        }
      }
    }
    for (auto& m : mine)
      for (int b : ev[m.first].places) loads[b].push_back(m.second);
  }
  for (int w = 0; w < (int)waves.size(); ++w) {
    const auto& ev = waves[w].ev;
    r.barriers = std::max<long>(r.barriers, waves[w].barriers);
    for (int i = 0; i < (int)ev.size(); ++i) {
      if (ev[i].kind != trace::READ) continue;
      int done = i + 1;  // the wait that covers this read
      while (done < (int)ev.size() && !(ev[done].kind == trace::LGKM && ev[done].n == 0)) ++done;
      const int done_barriers = done < (int)ev.size() ? ev[done].barriers : NEVER;
      for (int b : ev[i].places) {
        bool loaded = false;
        for (const Load& l : loads[b]) {
          ++r.pairs;
          const bool same = l.wave == w;
          const bool before = same ? l.waited_index < i : l.waited < NEVER && l.waited + 1 <= ev[i].barriers;
          const bool after = same ? l.index > done : done_barriers < NEVER && l.issued >= done_barriers + 1;
          loaded = loaded || before;
          if (before || after) continue;
          if (!r.races++) {
            char s[200];
            snprintf(s, sizeof s, "wave %d reads byte %d after %d barriers, waited for after %d; wave %d loads it after %d", w,
                     b * 64, ev[i].barriers, done_barriers, l.wave, l.issued);
            r.first = s;
          }
        }
        if (!loads[b].empty() && !loaded && b * 64 < free) ++r.unloaded;
      }
    }
  }
  return r;
}

template <class Kernel>
void run(const char* name, Kernel kernel, int waves, int blocks, int M, int N, int K, int out_bytes,
         long free = 1L << 30) {
  Fp8Problem p;
  const int kb = fp8_k_blocks(K);
  p.x = p.xs = p.w = p.ws = (const uint8_t*)(1L << 40);  // never read: recorded alone
  std::vector<float> b(N + 16, 0.f);
  p.bias = b.data();
  p.bias_f32 = 1;
  std::vector<char> y((size_t)M * N * out_bytes + 64);
  p.y = y.data();
  p.M = M;
  p.N = N;
  p.kb = kb;
  p.pitch = fp8_scale_pitch(K);
  // a first, short look for the array in LDS: its lowest load
  trace::Lane probe;
  trace::lane = &probe;
  trace::lds = trace::lds_end = nullptr;
  long lo = -1, hi = 0;
  blockIdx = dim3(0, 0, 0);
  gridDim = dim3(blocks);
  for (int w = 0; w < waves; ++w) {
    probe.ev.clear();
    threadIdx = dim3(w * 64, 0, 0);
    kernel(p);
    for (const auto& e : probe.ev)
      if (e.kind == trace::LOAD) {
        lo = lo < 0 ? e.at : std::min(lo, e.at);
        hi = std::max(hi, e.at + 64L * e.n);
      }
  }
  trace::lds = (char*)lo;
  trace::lds_end = (char*)hi;
  const Result r = check(record(kernel, p, waves, blocks), free);
  printf("%s M %d N %d K %d: loads %ld barriers %ld pairs %ld unloaded %ld races %ld %s\n", name, M, N, K, r.loads,
         r.barriers, r.pairs, r.unloaded, r.races, r.first.c_str());
}

}  // namespace
}  // namespace dit

int main() {
  using namespace dit;
  CASES
  return 0;
}
"""


def _run(tmp_path, cases, edit=lambda s: s):
    """The program's lines, one a case; edit: changes the kernels' source first, to see that the check sees it."""
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(RUNTIME)
    source = edit(open(os.path.join(CSRC, "gemm_fp8.hip")).read())
    source = source.replace('#include "device_common.h"', f'#include "{CSRC}/device_common.h"')
    (tmp_path / "kernels.h").write_text(source)
    src, exe = tmp_path / "run.cpp", tmp_path / "run"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "hip/hip_runtime.h"\n'
                   + MAIN.replace("SOURCE", str(tmp_path / "kernels.h")).replace("CASES", cases))
    r = subprocess.run([CLANG, "-O1", "-std=c++17", "-w", "-I", str(tmp_path), str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout.splitlines()


def _counts(line):
    w = line.split()
    return {k: int(w[w.index(k) + 1]) for k in ("loads", "barriers", "pairs", "unloaded", "races")}


needs_clang = pytest.mark.skipif(CLANG is None, reason="no clang++")

# 24 tiles, of which the block takes three (two of them whole, so that its waits count stores); every remainder of the
# K tiles by the four of a word of scales
CASES_256 = "\n".join(f'run("256x256", fp8_256_kernel, 8, 1, 6100, {n}, {k}, 2, 2 * 65536 + 2 * 2048);'
                      for k, n in ((384, 256), (500, 256), (640, 250), (700, 256), (900, 256), (1100, 256)))


@needs_clang
def test_places_of_the_256x256_kernel_are_read_before_they_are_loaded_again(tmp_path):
    lines = _run(tmp_path, CASES_256)
    assert len(lines) == 6
    for line in lines:
        c = _counts(line)
        assert c["loads"] > 500 and c["barriers"] > 90 and c["pairs"] > 10000, line
        assert c["races"] == 0 and c["unloaded"] == 0, line


CASES_SMALL = "\n".join(
    f'run("{cfg}", {kernel}, {waves}, {blocks}, {M}, {N}, {K}, {4 if "true" in kernel else 2});'
    for cfg, kernel, waves, blocks, M, N in (
        ("64x64", "fp8_ring_kernel<{f}, 64, 64, 2, 2, 2, {st}>", 8, 4, 100, 128),
        ("128x128", "fp8_ring_kernel<{f}, 128, 128, 2, 4, 1, {st}>", 8, 2, 200, 128),
        ("16x32", "fp8_split_kernel<{f}, 1, 2, 4>", 4, 2, 30, 32),
        ("32x32", "fp8_split_kernel<{f}, 2, 2, 4>", 4, 2, 60, 32),
        ("32x64", "fp8_split_kernel<{f}, 2, 4, 4>", 4, 2, 60, 64))
    for f in ("false", "true") for st in ((2, 4) if "st" in kernel else (0,)) if not (f == "true" and st == 4)
    for K in (100, 1280, 1700) for kernel in [f"({kernel.format(f=f, st=st)})"])


@needs_clang
def test_places_of_the_smaller_tiles_are_read_before_they_are_loaded_again(tmp_path):
    lines = _run(tmp_path, CASES_SMALL)
    assert len(lines) == 36
    for line in lines:
        c = _counts(line)
        assert c["loads"] > 0 and c["pairs"] > 0 and c["races"] == 0 and c["unloaded"] == 0, line


@needs_clang
@pytest.mark.parametrize("was,now", [
    ("wait_vmcnt<10>();  //", "wait_vmcnt<12>();  //"),                                          # ahead of the loop
    ("else wait_vmcnt<10>();", "else wait_vmcnt<12>();"),                                        # in a phase
    ("wait_vmcnt<10 + (STORE == 1", "wait_vmcnt<12 + (STORE == 1"),                              # beside the stores
    ("__builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)\n    const int byte", "const int byte"),  # for reads
    ("using CW = std::integral_constant<int, (c + Q - 2) % Q>", "using CW = std::integral_constant<int, (c + Q - 1) % Q>"),
])
def test_the_check_sees_what_comes_too_early(tmp_path, was, now):
    def edit(s):
        assert s.count(was) == 1
        return s.replace(was, now)
    lines = _run(tmp_path, CASES_256, edit)
    assert any(_counts(line)["races"] > 0 for line in lines), lines
