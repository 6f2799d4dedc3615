"""The 8-bit products', the quantising's and the block-sparse attention's kernels as
compiled for gfx950: LDS accesses in flight at block barriers, the stores that counted
waits count, and the registers and LDS on which launch rules count."""
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_isa_barriers_cpu import HIPCC, _compile, barriers_with_lds_in_flight

SOURCES = ["attention_sparse.hip", "gemm_fp8.hip", "quant_fp8.hip"]
LDS = 160 * 1024   # of a CU
SIMD = 512         # vector registers per lane of a SIMD


@pytest.fixture(scope="module")
def listings():
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(_compile, SOURCES)))


def _kernel(asm, name):
    """Instructions of the one kernel whose symbol matches."""
    lines = asm.splitlines()
    starts = [i for i, line in enumerate(lines) if re.match(r"^_Z\w*" + name + r"\w*:", line)]
    assert len(starts) == 1, (name, len(starts))
    end = next(j for j in range(starts[0], len(lines)) if "s_endpgm" in lines[j])
    return [t for t in (line.split(";")[0].strip() for line in lines[starts[0] + 1:end]) if t]


def reads_crossing_barriers(ins, most):
    """Barriers at which an LDS read issued more than `most` barriers before is still waited for, in program order."""
    flight, bad = [], []
    for n, t in enumerate(ins):
        if t.startswith("ds_read"):
            flight.append(0)
        c = re.search(r"lgkmcnt\((\d+)\)", t) if t.startswith("s_waitcnt") else None
        if c:
            flight = flight[len(flight) - int(c.group(1)):] if int(c.group(1)) else []
        if t == "s_barrier":
            flight = [x + 1 for x in flight]
            if any(x > most for x in flight):
                bad.append(n)
    return bad


def test_no_lds_access_in_flight_at_block_barriers(listings):
    """All kernels but the 256x256 one, whose reads end a turn later (test_lds_schedule_cpu.py checks their order)."""
    for src in SOURCES:
        assert "s_barrier" in listings[src], src
        bad = [b for b in barriers_with_lds_in_flight(listings[src]) if "fp8_256_kernel" not in b[0]]
        assert not bad, (src, bad[:8])


def test_reads_of_the_256x256_kernel_end_ahead_of_the_next_phases_barrier(listings):
    """A phase has two barriers: what it reads is waited for ahead of a third.  (But for the barrier behind the last
    phase, past which nothing is loaded.)"""
    ins = _kernel(listings["gemm_fp8.hip"], "fp8_256_kernel")
    last = len(ins) - 1 - ins[::-1].index("s_barrier")
    assert sum(t.startswith("ds_read_b128") for t in ins) > 100 and ins.count("s_barrier") > 30
    assert not any("lds" in t.split()[1:] for t in ins[last:])
    assert reads_crossing_barriers(ins[:last], 2) == []
    phase = ["ds_read_b128 v[0:3], v4", "s_waitcnt vmcnt(10)", "s_barrier", "s_barrier"]
    assert reads_crossing_barriers(phase + ["s_waitcnt lgkmcnt(0)", "s_barrier"], 2) == []
    assert reads_crossing_barriers(phase + ["s_barrier"], 2) == [4]
    assert reads_crossing_barriers(phase[:1] + phase + ["s_waitcnt lgkmcnt(1)", "s_barrier"], 2) == [6]


def test_a_phase_of_the_256x256_kernel_stores_as_often_as_its_waits_count(listings):
    """Between two barriers of the K tile that writes the sums of the tile before: four 16-byte stores, and otherwise
    only the elements of ragged rows, which no counted wait relies on.  The last tile's sums: sixteen."""
    parts, now = [], []
    for t in _kernel(listings["gemm_fp8.hip"], "fp8_256_kernel"):
        if t == "s_barrier":
            parts.append(now)
            now = []
        elif t.startswith(("global_store", "buffer_store", "flat_store")):
            now.append(t.split()[0])
    parts.append(now)
    # blocks of ragged rows are moved behind the kernel's straight path, so elements may follow the last tile's stores
    wide = [p.count("global_store_dwordx4") for p in parts]
    assert [n for n in wide if n] == [4, 4, 4, 4, 16], wide
    assert {op for p in parts for op in p} <= {"global_store_dwordx4", "global_store_short", "global_store_short_d16_hi"}


def _resources(asm):
    out, name = {}, None
    for line in asm.splitlines():
        m = re.match(r"^(_Z\w+):", line)
        if m:
            name = m.group(1)
        m = re.match(r"^; (TotalNumVgprs|ScratchSize|LDSByteSize): (\d+)", line)
        if m and name:
            out.setdefault(name, {})[m.group(1)] = int(m.group(2))
    return out


# kernel (its symbol), waves of a block, blocks that a CU must hold at a time
RESIDENT = [
    ("gemm_fp8.hip", "fp8_256_kernel", 8, 1),
    ("gemm_fp8.hip", "fp8_rows_kernelILb1E", 8, 4), ("gemm_fp8.hip", "fp8_rows_kernelILb0E", 8, 4),
    ("gemm_fp8.hip", "fp8_ring_kernelILb1ELi64ELi64ELi2ELi2ELi2ELi2E", 8, 2),
    ("gemm_fp8.hip", "fp8_ring_kernelILb0ELi64ELi64ELi2ELi2ELi2ELi2E", 8, 2),
    ("gemm_fp8.hip", "fp8_ring_kernelILb1ELi128ELi128ELi2ELi4ELi1ELi2E", 8, 2),
    ("gemm_fp8.hip", "fp8_ring_kernelILb0ELi128ELi128ELi2ELi4ELi1ELi2E", 8, 2),
    ("attention_sparse.hip", "sparse_bf16_kernelILi64ELi1E", 4, 3), ("attention_sparse.hip", "sparse_bf16_kernelILi128ELi1E", 4, 2),
    ("attention_sparse.hip", "sparse_bf16_kernelILi64ELi2E", 8, 1), ("attention_sparse.hip", "sparse_bf16_kernelILi128ELi2E", 8, 1),
    ("attention_sparse.hip", "select_blocks_kernelILi64ELi9ELi16ELi8E", 8, 2),
    ("attention_sparse.hip", "select_blocks_kernelILi128ELi9ELi16ELi8E", 8, 2),
]


def test_blocks_that_share_a_cu_fit_it(listings):
    res = {src: _resources(listings[src]) for src in SOURCES}
    for src, name, waves, blocks in RESIDENT:
        found = [v for k, v in res[src].items() if name in k]
        assert len(found) == 1, (name, len(found))
        r = found[0]
        per_simd = (waves * blocks + 3) // 4
        assert (r["TotalNumVgprs"] + 7) // 8 * 8 * per_simd <= SIMD, (name, r)
        assert r["LDSByteSize"] * blocks <= LDS, (name, r)


def test_no_kernel_spills(listings):
    for src in SOURCES:
        res = _resources(listings[src])
        assert res and all(r["ScratchSize"] == 0 for r in res.values()), src
