"""Post-build scan of the gfx950 assembly of libeqlinear.so.

The fp16 activation words are unpacked by one inline-asm statement per word
(``f16x2_to_f32`` in csrc/eql_common.h): a convert of the low half into an
early-clobber output, then a convert of the high half.  In some kernels this
toolchain's register allocator once gave that output the input's register (the
word then reads as already converted), and before the asm form, the same fault
showed as a word being overwritten between its two half-conversions.  A third
lost a whole element: the register of one tensor's was written by the unpack of
another tensor before it had been copied.  All of them give wrong numbers without any
error, so the build scans the device assembly for them and refuses to produce a library
that has one.

Checks, per kernel:
  clobbered_unpack   the unpack asm's first convert writes its own input register
  converted_source   an f16->f32 convert reads a register whose last write in
                     the same basic block was an fp32 result (a raw word is
                     never such a value), also by way of scratch memory
  lost_unpack        a result of the unpack asm that no path of the kernel
                     reads before its register is written again: an element
                     that another tensor's unpack took the register of
  mfma_dst_overlap   an MFMA whose result spans more than four registers has a
                     destination that partially overlaps its accumulator
                     input (srcC).  The gfx950 assembler refuses exactly this
                     form ("source 2 operand must not partially overlap with
                     dst") and accepts partial overlap for four-register
                     results, which the compiler emits for the 16x16 MFMAs
                     of these kernels; the check keeps a build from carrying
                     the refused form in code that bypassed the assembler's
                     operand validation.
  fused_scratch      a single-pass backward kernel (eql_bwd_fused_kernel) uses
                     scratch memory: only variants that fit the registers are
                     built, and a spilling one would run far slower than the
                     two-kernel path the host would otherwise have chosen.
"""
from __future__ import annotations

import glob
import os
import re
import subprocess

_FUNC = re.compile(r"^(_Z\S+):")
_BLOCK_END = re.compile(r"^\.LBB|^\s*s_cbranch|^\s*s_branch|^; %bb")
_CVT = re.compile(r"^\s*v_cvt_f32_f16\S*\s+v(\d+),\s*v(\d+)\b")
_F32_DEF = re.compile(r"^\s*(v_cvt_f32_f16\S*|v_add_f32\S*|v_sub_f32\S*|v_subrev_f32\S*|v_mul_f32\S*"
                      r"|v_fma_f32\S*|v_fmac_f32\S*|v_fmamk_f32\S*|v_fmaak_f32\S*)\s+v(\d+),")
_DEF_RANGE = re.compile(r"^\s*(v_\S+|buffer_load\S*|global_load\S*|scratch_load\S*|ds_read\S*)\s+v\[(\d+):(\d+)\]")
_DEF_ONE = re.compile(r"^\s*(v_\S+|buffer_load\S*|global_load\S*|scratch_load\S*|ds_read\S*)\s+v(\d+)\b")
_UNPACK_FIRST = re.compile(r"^\s*v_cvt_f32_f16_e32 v(\d+), v(\d+)\s*$")
_SCRATCH = re.compile(r"^; ScratchSize: (\d+)")
_SPILL = re.compile(r"^\s*scratch_(store|load)_dword(?:x\d)?\s+(?:off,\s*)?v(?:\[(\d+):(\d+)\]|(\d+)),\s*(?:off,\s*)?(\S+?)"
                    r"(?:\s+offset:(\d+))?\s*(?:;.*)?$")
_MFMA = re.compile(r"^\s*v_mfma\S*\s+([va])\[(\d+):(\d+)\],\s*[^,]+,\s*[^,]+,\s*([va])\[(\d+):(\d+)\]")


def scan_lines(lines):
    """Return a list of (kernel, check, instruction) problems found in assembly lines."""
    lines = list(lines)
    problems = []
    kernel = None
    last = {}          # vgpr -> "f32" | "other", within the current basic block
    slots = {}         # word of scratch memory -> the same
    in_asm = False
    asm_first = False
    for line in lines:
        m = _FUNC.match(line)
        if m:
            kernel, last, slots, in_asm = m.group(1), {}, {}, False
            continue
        if "ASMSTART" in line:
            in_asm, asm_first = True, True
            continue
        if "ASMEND" in line:
            in_asm = False
            continue
        sc = _SCRATCH.match(line)
        if sc and kernel and "eql_bwd_fused_kernel" in kernel and int(sc.group(1)) > 0:
            problems.append((kernel, "fused_scratch", line.strip()))
            continue
        if _BLOCK_END.match(line):
            last, slots = {}, {}
            continue
        if in_asm and asm_first:
            asm_first = False
            u = _UNPACK_FIRST.match(line)
            if u and u.group(1) == u.group(2):
                problems.append((kernel, "clobbered_unpack", line.strip()))
        mf = _MFMA.match(line)
        if mf:
            d0, d1, c0, c1 = (int(mf.group(i)) for i in (2, 3, 5, 6))
            if (mf.group(1) == mf.group(4) and d1 - d0 + 1 > 4 and (d0, d1) != (c0, c1)
                    and d0 <= c1 and c0 <= d1):
                problems.append((kernel, "mfma_dst_overlap", line.strip()))
        sp = _SPILL.match(line)
        if sp:
            first = int(sp.group(2) or sp.group(4))
            for k in range(first, int(sp.group(3) or sp.group(4)) + 1):
                slot = (sp.group(5), int(sp.group(6) or 0) + 4 * (k - first))
                if sp.group(1) == "store":
                    slots[slot] = last.get(k, "other")
                else:
                    last[k] = slots.get(slot, "other")
            continue
        c = _CVT.match(line)
        if c and last.get(int(c.group(2))) == "f32":
            problems.append((kernel, "converted_source", line.strip()))
        f = _F32_DEF.match(line)
        if f:
            last[int(f.group(2))] = "f32"
            continue
        r = _DEF_RANGE.match(line)
        if r:
            for k in range(int(r.group(2)), int(r.group(3)) + 1):
                last[k] = "other"
            continue
        d = _DEF_ONE.match(line)
        if d and not line.strip().startswith("v_cmp"):
            last[int(d.group(2))] = "other"
    return problems + lost_unpacks(lines)


_LABEL = re.compile(r"^(\.LBB\S+):")
_INST = re.compile(r"^\s+([a-z]\w+)\s*(.*)$")
_VGPRS = re.compile(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b")
_NO_RESULT = ("buffer_store", "buffer_atomic", "global_store", "global_atomic", "flat_store", "flat_atomic", "scratch_store", "ds_write",
              "ds_add", "v_cmp", "v_readfirstlane", "v_readlane", "s_")
_READS_RESULT = re.compile(r"fmac|dot|swap|writelane|dpp|UNUSED_PRESERVE|quad_perm|row_")
_ALL = (1 << 512) - 1


def _registers(operands) -> int:
    bits = 0
    for a, b, one in _VGPRS.findall(operands):
        bits |= 1 << int(one) if one else ((1 << (int(b) - int(a) + 1)) - 1) << int(a)
    return bits


def _written_and_read(op, operands):
    """VGPRs that an instruction writes and those that it reads, as bits."""
    if op in ("s_swappc_b64", "s_setpc_b64"):
        return 0, _ALL
    if op.startswith(_NO_RESULT):
        return 0, _registers(operands)
    first, _, others = operands.partition(",")
    written, read = _registers(first), _registers(others)
    if _READS_RESULT.search(op) or _READS_RESULT.search(operands):
        read |= written
    if "swap" in op:
        written |= read
    if "load_lds" in op or (op.startswith("buffer_load") and operands.endswith(" lds")):  # (the first operand is an address)
        written, read = 0, read | written
    return written, read


def lost_unpacks(lines):
    """(kernel, "lost_unpack", instruction) for each conversion of an unpack asm whose result is dead: liveness over the
    kernel's basic blocks, from s_endpgm back."""
    problems, kernel, body = [], None, []
    for line in lines:
        m = _FUNC.match(line)
        if m or line.startswith(".Lfunc_end"):
            problems += _lost(kernel, body)
            kernel, body = m.group(1) if m else None, []
        elif kernel:
            body.append(line)
    return problems + _lost(kernel, body)


def _lost(kernel, body):
    if not any("ASMSTART" in line for line in body):
        return []
    blocks, ends, label, block, in_asm = [], [], {}, [], False
    for line in body:
        m = _LABEL.match(line)
        if "ASMSTART" in line or "ASMEND" in line:
            in_asm = "ASMSTART" in line
            continue
        inst = None if m else _INST.match(line.split(";")[0])
        op, operands = (inst.group(1), inst.group(2).strip()) if inst else ("", "")
        if m or op == "s_branch" or op.startswith("s_cbranch") or op == "s_endpgm":
            blocks.append(block)
            ends.append((op, operands))
            block = []
            if m:
                label[m.group(1)] = len(blocks)
        elif op:
            block.append((*_written_and_read(op, operands), in_asm and op.startswith("v_cvt_f32_f16"), line))
    blocks.append(block)
    ends.append(("", ""))
    after = len(blocks)  # what follows the text, and labels outside it: everything may be read there
    succ = [() if op == "s_endpgm" else (label.get(to, after),) if op == "s_branch" else (i + 1, label.get(to, after)) if op else (i + 1,)
            for i, (op, to) in enumerate(ends)]
    use, kill = [], []
    for b in blocks:
        u = k = 0
        for written, read, _, _ in b:
            u |= read & ~k
            k |= written
        use.append(u)
        kill.append(k)
    live, changed = [0] * after + [_ALL], True

    def out(i):
        bits = 0
        for s in succ[i]:
            bits |= live[s]
        return bits

    while changed:
        changed = False
        for i in range(after - 1, -1, -1):
            bits = use[i] | (out(i) & ~kill[i])
            changed, live[i] = changed or bits != live[i], bits
    problems = []
    for i, b in enumerate(blocks):
        bits = out(i)
        for written, read, unpack, line in reversed(b):
            if unpack and not bits & written:
                problems.append((kernel, "lost_unpack", line.strip()))
            bits = (bits & ~written) | read
    return problems


def scan_file(path):
    with open(path) as f:
        return scan_lines(f)


def device_asm_files(build_dir):
    return sorted(glob.glob(os.path.join(build_dir, "**", "*-hip-amdgcn-amd-amdhsa-*.s"), recursive=True))


def demangle(names):
    try:
        out = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True).stdout
        return out.split("\n")[: len(names)]
    except OSError:
        return list(names)


def check_build(build_dir):
    """Scan every device assembly file of a build; raise RuntimeError on a problem."""
    files = device_asm_files(build_dir)
    if not files:
        raise RuntimeError("no device assembly found in %s (the build keeps it with -save-temps)" % build_dir)
    problems = []
    for path in files:
        problems += [(os.path.basename(path),) + p for p in scan_file(path)]
    if problems:
        names = demangle([p[1] for p in problems])
        msg = "\n".join("  %s: %s: %s: %s" % (p[0], n, p[2], p[3]) for p, n in zip(problems[:20], names))
        raise RuntimeError("device code failed the post-build check (%d findings):\n%s"
                           % (len(problems), msg))
    return files
