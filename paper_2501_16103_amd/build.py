"""Compile the HIP sources into libmoe_sb.so (gfx950 only), in-tree."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(HERE, "libmoe_sb.so")
SRCS = [os.path.join(HERE, "csrc", f) for f in ("moe_sb.hip", "moe_mx4.hip")]
# measurement kernels, kept out of the product library
PROBE_LIB = os.path.join(HERE, "libmoe_probe.so")
PROBE_SRCS = [os.path.join(HERE, "csrc", "moe_probe.hip")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-FP32 instructions are switched off for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # The k loops are unrolled completely by pragma; at the default size limit for pragma-unrolled loops the largest
    # copies sit at the edge, and a loop left rolled indexes the accumulators dynamically, which puts them in memory.
    "-mllvm", "-pragma-unroll-threshold=100000",
]


# A register spill inside a k loop is a vector memory instruction among the hand-counted global->LDS DMAs: the
# compiler waits for its reload with vmcnt(0), which drains the whole DMA ring every iteration (measured: a
# third of the throughput gone).  The build therefore reads the device assembly and refuses a GEMM kernel that
# has a scratch access inside a loop that also holds MFMAs.  (Spills outside the loops only cost their own time;
# they cannot let a DMA wait pass early: loads retire in order and extra entries in vmcnt make a wait stricter.)
# The 4-bit products and the layer for few tokens are held to the same: their loops over k, of fewer MFMAs a step, have loads of
# later steps under way, which the wait for a reload drains as well.
SPILL_CHECKED = "(?:gemm|few_tokens)"


def check_no_spill_in_k_loops(asm_text: str) -> None:
    # accumulators or fragments that were not promoted to registers show up as a large private segment
    for m in re.finditer(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", asm_text):
        if re.search(SPILL_CHECKED, m.group(1)) and int(m.group(2)) > 256:
            raise RuntimeError(f"{m.group(1)}: {m.group(2)} bytes of private memory per lane (an array left in memory?)")
    for m in re.finditer(rf"^(_ZN3moe\S*{SPILL_CHECKED}\S*):\s*(?:;.*)?$", asm_text, re.M):
        name = m.group(1)
        least = 4 if "mx4_gemm" in name or "few_tokens" in name else 16   # MFMAs of a k-step
        end = asm_text.find(".Lfunc_end", m.end())
        lines = asm_text[m.end():end].splitlines()
        label_at = {ln.split(":")[0]: k for k, ln in enumerate(lines) if ln.startswith(".LBB")}
        loops = []   # (first line, last line) of every backward branch's span

        def exits(k):   # the block at line k does nothing but end the program (an early-placed exit, not a loop head)
            for ln in lines[k + 1:]:
                ln = ln.strip()
                if ln and not ln.startswith(";"):
                    return ln.startswith("s_endpgm")
            return False

        for k, ln in enumerate(lines):
            b = re.search(r"s_cbranch\w*\s+(\.LBB\d+_\d+)", ln)
            if b and label_at.get(b.group(1), len(lines)) < k and not exits(label_at[b.group(1)]):
                loops.append((label_at[b.group(1)], k))
        def mfmas(lo, hi):
            return sum("v_mfma" in lines[x] for x in range(lo, hi + 1))

        for k, ln in enumerate(lines):
            if "scratch_" not in ln:
                continue
            around = [lp for lp in loops if lp[0] <= k <= lp[1]]
            if not around:
                continue
            lo, hi = min(around, key=lambda lp: lp[1] - lp[0])          # the innermost loop around the access
            inner = [lp for lp in loops if lo <= lp[0] and lp[1] <= hi and lp != (lo, hi)]
            if any(mfmas(a, b) >= least for a, b in inner):
                # a loop over tiles (resident kernels) with the k loops inside it: a reload between two tiles costs
                # its own time only -- unless it sits in the middle of a straight run of MFMAs (the unrolled last
                # iterations of a tile, which still have DMAs in flight)
                if mfmas(max(lo, k - 40), k) >= least // 2 and mfmas(k, min(hi, k + 40)) >= least // 2:
                    raise RuntimeError(f"{name}: register spill among the MFMAs of a tile's last iterations")
                continue
            own = sum("v_mfma" in lines[x] for x in range(lo, hi + 1) if not any(a <= x <= b for a, b in inner))
            if own >= least:
                raise RuntimeError(f"{name}: register spill inside a k loop (it would drain the DMA ring every iteration)")


# MFMAs of the alternating-role loops are written out, so the compiler does not know them and keeps no distance between an
# ordinary vector instruction and an MFMA that reads its result (two wait states on gfx950; it does so around its own).
# The build refuses a GEMM kernel where such an MFMA follows the write of one of its operands too closely on any path.
MFMA_READ_WAIT_STATES = 2


def _registers(operand: str) -> set:
    m = re.fullmatch(r"([va])(?:(\d+)|\[(\d+):(\d+)\])", operand.strip())
    if not m:
        return set()
    lo, hi = (m.group(2), m.group(2)) if m.group(2) else (m.group(3), m.group(4))
    return {(m.group(1), r) for r in range(int(lo), int(hi) + 1)}


def check_mfma_operand_distance(asm_text: str) -> None:
    for m in re.finditer(r"^(_ZN3moe\S*gemm\S*):\s*(?:;.*)?$", asm_text, re.M):
        name = m.group(1)
        code = []   # (is a label, text, written out by hand)
        in_asm = False
        for ln in asm_text[m.end():asm_text.find(".Lfunc_end", m.end())].splitlines():
            if "#ASMSTART" in ln or "#ASMEND" in ln:
                in_asm = "#ASMSTART" in ln
                continue
            text = ln.split(";")[0].strip()
            label = re.match(r"(\.LBB\S+):", text)
            if label:
                code.append((True, label.group(1), False))
            elif re.match(r"[a-z]+_", text):
                code.append((False, text, in_asm))
        branches_to = {}
        for k, (is_label, text, _) in enumerate(code):
            b = re.match(r"s_c?branch\S*\s+(\.LBB\S+)", text)
            if b and not is_label:
                branches_to.setdefault(b.group(1), []).append(k)

        def before(k):   # the lines that can run just before line k
            prev = [k - 1] if k > 0 and not re.match(r"s_(branch|endpgm|setpc_b64)\b", code[k - 1][1]) else []
            return prev + (branches_to.get(code[k][1], []) if code[k][0] else [])

        for k, (is_label, text, by_hand) in enumerate(code):
            if is_label or not by_hand or not text.startswith("v_mfma"):
                continue
            # A, B, C and, of a scaled one, the two registers of scales (modifiers follow the last operand behind a blank)
            operands = text.split(None, 1)[1].split(",")[1:6 if text.startswith("v_mfma_scale") else 4]
            reads = set().union(*(_registers(op.split()[0]) for op in operands))
            todo, seen = [(p, 0) for p in before(k)], set()
            while todo:
                p, waited = todo.pop()
                if waited >= MFMA_READ_WAIT_STATES or (p, waited) in seen:
                    continue
                seen.add((p, waited))
                p_label, p_text, _ = code[p]
                if not p_label:
                    operands = p_text.split(None, 1)[1].split(",") if " " in p_text else []
                    written = set().union(*(_registers(op) for op in operands[:2 if p_text.startswith("v_swap") else 1]))
                    if p_text.startswith("v_") and not p_text.startswith("v_mfma") and written & reads:
                        raise RuntimeError(f"{name}: '{text}' {waited} wait states behind '{p_text}'")
                    nop = re.match(r"s_nop\s+(\d+)", p_text)
                    waited += int(nop.group(1)) + 1 if nop else 1
                todo += [(q, waited) for q in before(p)]


def _compile(srcs: list, lib: str, check_asm: bool, verbose: bool) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        jobs = []
        for src in srcs:   # side by side, each in a folder of its own for the files it leaves
            out = os.path.join(tmp, os.path.splitext(os.path.basename(src))[0])
            os.mkdir(out)
            cmd = [hipcc] + HIPCC_FLAGS + ["-save-temps=obj", "-c", src, "-o", os.path.join(out, "out.o")]
            jobs.append((out, cmd, subprocess.Popen(cmd, cwd=out, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        logs = [job.communicate()[0] for _, _, job in jobs]   # (all of them end before the folder goes)
        for (out, cmd, job), log in zip(jobs, logs):
            if job.returncode != 0:
                raise RuntimeError("hipcc failed:\n" + log)
            if check_asm:
                asm = [f for f in os.listdir(out) if f.endswith(".s") and "amdgcn" in f]
                if not asm:
                    raise RuntimeError("no device assembly found next to the object file")
                with open(os.path.join(out, asm[0])) as f:
                    asm_text = f.read()
                check_no_spill_in_k_loops(asm_text)
                check_mfma_operand_distance(asm_text)
            if verbose:
                print(" ".join(cmd))
        linked = os.path.join(tmp, os.path.basename(lib))
        cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + [os.path.join(out, "out.o") for out, _, _ in jobs] + ["-o", linked]
        res = subprocess.run(cmd, cwd=tmp, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("linking failed:\n" + res.stdout + res.stderr)
        shutil.copyfile(linked, lib)
        os.chmod(lib, 0o755)
    return lib


def build_library(verbose: bool = False) -> str:
    """libmoe_sb.so: the product library."""
    return _compile(SRCS, LIB, True, verbose)


def build_probe_library(verbose: bool = False) -> str:
    """libmoe_probe.so: the measurement kernels (bench.py --mfma-probe and two tests load it)."""
    return _compile(PROBE_SRCS, PROBE_LIB, False, verbose)


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_probe_library(verbose=True))
