"""The 4-bit products', the rotary positions' and the grouped attention's kernels as compiled for gfx950: LDS accesses in
flight at block barriers, the stores that counted waits count, what instructions written as statements need around them,
and the registers and LDS on which launch rules count."""
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_isa_barriers_cpu import HIPCC, _compile, barriers_with_lds_in_flight
from test_lowbit_listings_cpu import LDS, SIMD, _kernel, _resources

SOURCES = ["attention_grouped.hip", "gemm_fp4.hip", "quant_fp4.hip", "rope.hip"]


@pytest.fixture(scope="module")
def listings():
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(_compile, SOURCES)))


def test_no_lds_access_in_flight_at_block_barriers(listings):
    assert all("s_barrier" in listings[src] for src in SOURCES[:2])
    for src in SOURCES:
        bad = barriers_with_lds_in_flight(listings[src])
        assert not bad, (src, bad[:8])


def test_no_kernel_spills(listings):
    for src in SOURCES:
        res = _resources(listings[src])
        assert res and all(r["ScratchSize"] == 0 for r in res.values()), src


@pytest.mark.parametrize("f32,per_phase", [(0, 8), (1, 16)])
def test_a_phase_of_the_256x256_kernel_stores_as_often_as_its_waits_count(listings, f32, per_phase):
    """Between two barriers of the phases that write rows of sums, 16-byte stores; the last tile's rows 1 to 3 behind the
    last barrier."""
    parts, now = [], []
    for t in _kernel(listings["gemm_fp4.hip"], f"fp4_256_kernelILb{f32}E"):
        if t == "s_barrier":
            parts.append(now)
            now = []
        elif t.startswith(("global_store", "buffer_store", "flat_store")):
            now.append(t.split()[0])
    parts.append(now)
    wide = [p.count("global_store_dwordx4") for p in parts]
    assert sorted(n for n in wide if n) == [per_phase] * 4 + [3 * per_phase], wide
    narrow = {op for p in parts for op in p} - {"global_store_dwordx4"}
    assert narrow <= ({"global_store_dword", "global_store_dwordx2", "global_store_dwordx3"} if f32
                      else {"global_store_short", "global_store_short_d16_hi"}), narrow


MFMA = re.compile(r"v_mfma_scale_f32_32x32x64_f8f6f4 a\[(\d+):(\d+)\], v\[(\d+):(\d+)\], v\[(\d+):(\d+)\], \S+ v(\d+), v(\d+)")
READ_AFTER = 19   # wait states between a 16-pass product and a vector instruction's read of its sums
PASSES = 8        # of this one, for which it holds the issue of the next


def _registers(operands, kind):
    out = set()
    for m in re.finditer(rf"\b{kind}(?:(\d+)\b|\[(\d+):(\d+)\])", operands):
        out |= {int(m.group(1))} if m.group(1) else set(range(int(m.group(2)), int(m.group(3)) + 1))
    return out


def hazards(ins):
    """Products that read what one of the two instructions before writes, and reads of a product's sums that come too
    early, in program order."""
    bad, states, ready, written = [], 0, {}, []
    for n, t in enumerate(ins):
        if t.endswith(":"):
            continue
        if t == "s_barrier":
            ready, written = {}, []
        op, _, rest = t.partition(" ")
        m = MFMA.match(t)
        if m:
            g = [int(x) for x in m.groups()]
            reads = set(range(g[2], g[3] + 1)) | set(range(g[4], g[5] + 1)) | {g[6], g[7]}
            if any(w & reads for w in written[-2:]):
                bad.append((n, t))
            ready.update({a: states + READ_AFTER for a in range(g[0], g[1] + 1)})
            states += PASSES
            written.append(set())
            continue
        if op.startswith("v_") and any(states < ready.get(a, 0) for a in _registers(rest, "a")):
            bad.append((n, t))
        written.append(_registers(rest.split(",")[0], "v") if op.startswith("v_") and not op.startswith("v_cmp") else set())
        if op.startswith("v_permlane16_swap"):
            written[-1] = _registers(rest, "v")
        states += int(rest) + 1 if op == "s_nop" else 1
    return bad


@pytest.mark.parametrize("f32", [0, 1])
def test_statements_of_the_256x256_kernel_keep_their_distances(listings, f32):
    ins = _kernel(listings["gemm_fp4.hip"], f"fp4_256_kernelILb{f32}E")
    assert sum(bool(MFMA.match(t)) for t in ins) >= 16 * 8 * 3
    assert sum(t.startswith("v_accvgpr_read") for t in ins) >= 64 * 4
    assert hazards(ins) == []


def test_the_check_of_distances_sees_short_ones():
    mfma = "v_mfma_scale_f32_32x32x64_f8f6f4 a[0:15], v[0:3], v[4:7], a[0:15], v8, v9 op_sel:[0,0,0] cbsz:4 blgp:4"
    assert MFMA.match(mfma) and hazards([mfma]) == []
    assert len(hazards(["v_mov_b32_e32 v8, v20", mfma])) == 1
    assert len(hazards(["v_mov_b32_e32 v8, v20", "s_nop 0", mfma])) == 1
    assert hazards(["v_mov_b32_e32 v8, v20", "s_nop 0", "s_nop 0", mfma]) == []
    assert hazards(["v_mov_b32_e32 v21, v8", mfma]) == []
    assert len(hazards([mfma, "s_nop 7", "v_accvgpr_read_b32 v30, a3"])) == 1
    assert hazards([mfma, "s_nop 7", "s_nop 7", "v_accvgpr_read_b32 v30, a3"]) == []
    assert hazards([mfma, "s_nop 1", "v_accvgpr_read_b32 v30, a16"]) == []


# kernel (its symbol), waves of a block, blocks that a CU must hold at a time
RESIDENT = [
    ("gemm_fp4.hip", "fp4_256_kernelILb1E", 4, 1), ("gemm_fp4.hip", "fp4_256_kernelILb0E", 4, 1),
    ("gemm_fp4.hip", "fp4_rows_kernelILb1E", 8, 2), ("gemm_fp4.hip", "fp4_rows_kernelILb0E", 8, 2),
    ("gemm_fp4.hip", "fp4_ring_kernelILb1ELi64ELi64ELi2ELi2ELi2ELi2E", 8, 2),
    ("gemm_fp4.hip", "fp4_ring_kernelILb0ELi64ELi64ELi2ELi2ELi2ELi2E", 8, 2),
    ("gemm_fp4.hip", "fp4_ring_kernelILb1ELi128ELi128ELi2ELi4ELi1ELi2E", 8, 2),
    ("gemm_fp4.hip", "fp4_ring_kernelILb0ELi128ELi128ELi2ELi4ELi1ELi2E", 8, 2),
    ("attention_grouped.hip", "grouped_bf16_kernelILi64E", 4, 2), ("attention_grouped.hip", "grouped_bf16_kernelILi128E", 4, 2),
    ("attention_grouped.hip", "grouped_few_kernelILi64E", 4, 2), ("attention_grouped.hip", "grouped_few_kernelILi128E", 4, 2),
]


def test_blocks_that_share_a_cu_fit_it(listings):
    res = {src: _resources(listings[src]) for src in SOURCES}
    for src, name, waves, blocks in RESIDENT:
        found = [v for k, v in res[src].items() if name in k]
        assert found, name
        for r in found:
            per_simd = (waves * blocks + 3) // 4
            assert (r["TotalNumVgprs"] + 7) // 8 * 8 * per_simd <= SIMD, (name, r)
            assert r["LDSByteSize"] * blocks <= LDS, (name, r)
