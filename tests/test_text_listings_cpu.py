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


def _function(asm, name):
    """Instructions and labels of the kernel, those of blocks behind its first end among them."""
    lines = asm.splitlines()
    start = next(i for i, line in enumerate(lines) if re.match(r"^_Z\w*" + name + r"\w*:", line))
    end = next(j for j in range(start, len(lines)) if lines[j].startswith(".Lfunc_end"))
    code = [t for t in (line.split(";")[0].strip() for line in lines[start + 1:end]) if t]
    return [t for t in code if re.match(r"\.LBB\w+:$", t) or not t.startswith(".")]


def _blocks(ins):
    """Runs of instructions that begin at a label or behind a branch, and for each the runs that may follow it."""
    starts = sorted({0} | {n for n, t in enumerate(ins) if t.endswith(":")}
                    | {n + 1 for n, t in enumerate(ins) if t.startswith(("s_cbranch", "s_branch", "s_endpgm"))} - {len(ins)})
    at = {ins[n][:-1]: i for i, n in enumerate(starts) if ins[n].endswith(":")}
    runs, next_of = [], []
    for i, n in enumerate(starts):
        run = ins[n:starts[i + 1] if i + 1 < len(starts) else len(ins)]
        last = run[-1]
        follow = [at[last.split()[1]]] if last.startswith(("s_cbranch", "s_branch")) else []
        if not last.startswith(("s_branch", "s_endpgm")) and i + 1 < len(starts):
            follow.append(i + 1)
        runs.append([t for t in run if not t.endswith(":")])
        next_of.append(follow)
    return runs, next_of


OPERAND_AFTER = 2  # wait states between a vector instruction's write and a product's read


def _step(t, age):
    """What instruction t does too early, given the wait states since registers were written, and those behind it.
    age: (kind, number, by) -> states since, of vector instructions' writes ("w") and products' sums ("p")."""
    op, _, rest = t.partition(" ")
    bad, wrote = False, set()
    m = MFMA.match(t)
    if m:
        g = [int(x) for x in m.groups()]
        sums = {("a", a) for a in range(g[0], g[1] + 1)}
        reads = {("v", v) for v in [*range(g[2], g[3] + 1), *range(g[4], g[5] + 1), g[6], g[7]]} | sums
        bad = any(age.get((*r, "w"), OPERAND_AFTER) < OPERAND_AFTER for r in reads)
        wrote = {(*r, "p") for r in sums}
    else:
        used = {(kind, n) for kind in "av" for n in _registers(rest, kind)}
        bad = any(age.get((*r, "p"), READ_AFTER) < READ_AFTER for r in used)
        if op.startswith("v_") and not op.startswith("v_cmp"):
            first = rest if "swap" in op else rest.split(",")[0]
            wrote = {(kind, n, "w") for kind in "av" for n in _registers(first, kind)}
    states = int(rest) + 1 if op == "s_nop" else 1
    after = {r: n + states for r, n in age.items() if n + states < READ_AFTER}
    after.update({r: 0 for r in wrote})
    return bad, after


def too_early(ins):
    """Over every path: products that read what a vector instruction wrote less than OPERAND_AFTER wait states ago, their
    sums among it, and instructions of any kind, stores too, that touch a product's sums less than READ_AFTER behind it.
    Every instruction counts as one wait state, a barrier too, a product no more."""
    runs, next_of = _blocks(ins)
    entry, todo, bad = {0: {}}, [0], set()
    while todo:
        i = todo.pop()
        age = entry[i]
        for n, t in enumerate(runs[i]):
            early, age = _step(t, age)
            if early:
                bad.add((i, n, t))
        for j in next_of[i]:
            old = entry.get(j)
            new = age if old is None else {**age, **{r: min(n, age.get(r, n)) for r, n in old.items()}}
            if new != old:
                entry[j] = new
                todo.append(j)
    return sorted(bad)


@pytest.mark.parametrize("f32", [0, 1])
def test_statements_of_the_256x256_kernel_keep_their_distances_on_every_path(listings, f32):
    ins = _function(listings["gemm_fp4.hip"], f"fp4_256_kernelILb{f32}E")
    products = [t for t in ins if "mfma" in t]
    assert len(products) >= 16 * 8 * 3 and all(MFMA.match(t) for t in products)
    assert sum(t.startswith("v_accvgpr_") for t in ins) >= 64 * 4 and sum(t.startswith("s_endpgm") for t in ins) >= 1
    runs, next_of = _blocks(ins)
    seen, todo = {0}, [0]
    while todo:
        new = set(next_of[todo.pop()]) - seen
        seen |= new
        todo += new
    reached = [t for i in seen for t in runs[i]]
    assert sum(bool(MFMA.match(t)) for t in reached) == len(products)
    assert too_early(ins) == []


def test_the_check_of_paths_sees_short_distances():
    mfma = "v_mfma_scale_f32_32x32x64_f8f6f4 a[0:15], v[0:3], v[4:7], a[0:15], v8, v9 op_sel:[0,0,0] cbsz:4 blgp:4"
    first = mfma.replace("a[0:15], v8", "0, v8")
    wait = ["s_nop 7", "s_nop 7", "s_nop 1"]  # one state short
    early = lambda *ins: len(too_early(list(ins)))
    assert MFMA.match(first) and early(mfma, mfma) == 0
    # what a product reads, in front of a barrier too
    assert early("v_mov_b32_e32 v8, v20", mfma) == 1 and early("v_mov_b32_e32 v8, v20", "s_barrier", mfma) == 1
    assert early("v_mov_b32_e32 v8, v20", "s_nop 0", "s_barrier", mfma) == 0 == early("v_mov_b32_e32 v8, v20", "s_nop 1", mfma)
    assert early("v_permlane16_swap_b32 v30, v4", mfma) == 1 and early("v_mov_b32_e32 v21, v8", mfma) == 0
    # its sums ahead of it
    assert early("v_accvgpr_write_b32 a0, v3", mfma) == 1 and early("v_accvgpr_mov_b32 a7, a20", "s_barrier", first) == 1
    assert early("v_accvgpr_write_b32 a0, v3", "s_nop 1", mfma) == 0
    # its sums behind it: read, stored, written
    for use, other in (("v_accvgpr_read_b32 v30, a3", "v_accvgpr_read_b32 v30, a16"),
                       ("global_store_dwordx4 v[20:21], a[12:15], off nt", "global_store_dwordx4 v[20:21], a[16:19], off nt"),
                       ("ds_write_b128 v20, a[0:3]", "ds_write_b128 v20, a[16:19]"),
                       ("v_accvgpr_write_b32 a15, 0", "v_accvgpr_write_b32 a16, 0"),
                       ("v_accvgpr_mov_b32 a30, a1", "v_accvgpr_mov_b32 a30, a16")):
        assert early(mfma, "s_barrier", use) == 1 and early(mfma, *wait, use) == 1, use
        assert early(mfma, *wait, "s_barrier", use) == 0 and early(mfma, other) == 0, use
    # over a branch, and from the end of a loop to its start
    jump = [mfma, "s_cbranch_execz .LBB0_1", *wait, "s_nop 7", ".LBB0_1:", "v_accvgpr_read_b32 v30, a3"]
    assert early(*jump) == 1 and early(*(t for t in jump if "branch" not in t)) == 0
    loop = [".LBB0_1:", mfma, *wait, "s_nop 7", "v_mov_b32_e32 v8, v20", "s_cbranch_scc1 .LBB0_1", "s_endpgm"]
    assert early(*loop) == 1 and early(*(loop[:-2] + ["s_nop 0"] + loop[-2:])) == 0
    assert early(mfma, "s_branch .LBB0_2", "v_accvgpr_read_b32 v30, a3", ".LBB0_2:", *wait, "s_nop 0", "v_accvgpr_read_b32 v30, a3") == 0


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
