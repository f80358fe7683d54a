"""Compile the HIP library (csrc/*.hip) for gfx950 into paper_2511_17885_amd/libfmoe.so.

hipcc cross-compiles without a GPU.  Packed-fp32 instruction selection is disabled for all
device code; the router and pruning kernels are additionally built with floating-point
contraction off because their operation order is part of their contract.
"""
import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
OUT = os.path.join(HERE, "libfmoe.so")

COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-fast-math",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-function"]
SOURCES = {
    "api.hip": [],
    "route.hip": ["-ffp-contract=off"],
    "prune.hip": ["-ffp-contract=off"],
    "permute.hip": [],
    "ffn.hip": [],
    "ffn_quant.hip": [],
    "ffn_rows8.hip": [],
    "select.hip": [],
    "quant.hip": [],
    "norm.hip": ["-ffp-contract=off"],
    "combine.hip": [],
    "decode.hip": ["-ffp-contract=off"],
    "diag.hip": [],
    "stack.hip": [],
    "noalloc.hip": [],
}


HAND_PLACED = ("ffn.hip", "ffn_quant.hip", "ffn_rows8.hip")   # files whose kernels name accumulation registers themselves


def check_accumulation_registers(asm_path):
    """The dense-shape expert GEMM kernels (ffn_dense_kernel, ffn_quant_dense_kernel, ffn_rows8_many_kernel) keep their accumulators in accumulation
    registers that the kernel names itself, which the compiler's register allocator does not see.  This
    reads the device assembly the compiler wrote for their file and fails if, inside those kernels, the
    compiler placed anything of its own in an accumulation register (any a<N> operand outside the
    kernel's own inline-assembly blocks), or spilled a register (their LDS reads are inline assembly and
    land later than the compiler believes)."""
    import re
    inside = in_asm = False
    kernels = 0
    for n, line in enumerate(open(asm_path), 1):
        if re.match(r"^_ZN\S*(ffn_dense_kernel|ffn_quant_dense_kernel|ffn_rows8_many_kernel)\S*:", line):
            inside, in_asm = True, False
            kernels += 1
            name = line.split(":")[0]
            continue
        if not inside:
            continue
        if line.startswith(".Lfunc_end"):   # not s_endpgm: a kernel has one per early exit
            inside = False
        elif "ASMSTART" in line:
            in_asm = True
        elif "ASMEND" in line:
            in_asm = False
        elif "Spill" in line:
            raise RuntimeError(f"{asm_path}:{n}: the compiler spills a register inside {name}: {line.strip()}")
        elif not in_asm and re.search(r"\ba\[?\d", line.split(";")[0]):
            raise RuntimeError(f"{asm_path}:{n}: the compiler uses an accumulation register inside {name}, which "
                               f"keeps hand-placed accumulators there: {line.strip()}")
    if kernels == 0:
        raise RuntimeError(f"{asm_path}: no dense-shape kernel found to check")
    return kernels


def check_pending_reads(asm_path):
    """Some kernels start LDS reads in one inline-assembly block and wait for them in a later one; the compiler takes their
    registers as written at once.  This reads the device assembly and fails if an instruction of the compiler's own
    touches such a register before the wait."""
    import re

    def registers(text):
        found = set()
        for m in re.finditer(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
            lo = int(m.group(1) or m.group(3))
            found.update(range(lo, int(m.group(2) or lo) + 1))
        return found

    in_asm, pending, reads = False, set(), 0
    for n, line in enumerate(open(asm_path), 1):
        code = line.split(";")[0].strip()
        if "ASMSTART" in line:
            in_asm = True
        elif "ASMEND" in line:
            in_asm = False
        elif line.startswith(".Lfunc_end"):
            pending = set()
        elif code.startswith("s_waitcnt") and "lgkmcnt(0)" in code:
            pending = set()
        elif in_asm and code.startswith("ds_read"):
            pending |= registers(code.split(",")[0])
            reads += 1
        elif not in_asm and pending and code and not code.startswith(".") and registers(code) & pending:
            raise RuntimeError(f"{asm_path}:{n}: the compiler touches a register that an LDS read has not reached yet: {code}")
    return reads


def check_matrix_operands(asm_path):
    """A matrix instruction may read a register that a vector instruction has written only two waits later.  The compiler keeps to that with its
    own instructions, not with those in inline assembly.  This reads the device assembly and fails where such a write is nearer, on the way
    down or by a branch.  Exchanges (v_swap, v_permlane*_swap) write both of their operands."""
    import re

    def registers(text):
        found = set()
        for m in re.finditer(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
            lo = int(m.group(1) or m.group(3))
            found.update(range(lo, int(m.group(2) or lo) + 1))
        return frozenset(found)

    lines, in_asm = [], False   # (number, code, within inline assembly)
    for n, line in enumerate(open(asm_path), 1):
        code = line.split(";")[0].strip()
        if "ASMSTART" in line or "ASMEND" in line:
            in_asm = "ASMSTART" in line
        elif code.endswith(":") or (code and not code.startswith((".", "#"))):
            lines.append((n, code, in_asm))
    none = frozenset()
    entered, before = {}, None  # label -> what the last two instructions wrote, over the branches that lead there
    while entered != before:    # twice or three times: two instructions reach over two branches at most
        before, entered, seen, recent = entered, dict(entered), 0, (none, none)
        for n, code, in_asm in lines:
            word = code.split()[0]
            if code.endswith(":"):
                recent = tuple(a | b for a, b in zip(recent, before.get(code[:-1], (none, none))))
            elif word == "s_nop":
                recent = ((none,) * (int(code.split()[1], 0) + 1) + recent)[:2]
            elif word.startswith("v_mfma"):
                if in_asm:
                    seen += 1
                    if any(registers(code.split(",", 1)[1]) & r for r in recent):
                        raise RuntimeError(f"{asm_path}:{n}: a matrix instruction reads a register that was written just before it: {code}")
                recent = (none, recent[0])
            elif word.startswith(("s_branch", "s_cbranch")):
                recent, label = (none, recent[0]), code.split()[-1]
                entered[label] = tuple(a | b for a, b in zip(recent, entered.get(label, (none, none))))
                if word == "s_branch":
                    recent = (none, none)
            elif word in ("s_endpgm", "s_setpc_b64"):
                recent = (none, none)
            else:
                operands = code[len(word):].split(",")
                written = none
                if word.startswith("v_") and not word.startswith("v_cmp"):
                    written = registers(",".join(operands[:2 if "swap" in word else 1]))
                recent = (written, recent[0])
    return seen


def _compile(name, extra, verbose):
    src = os.path.join(CSRC, name)
    obj = os.path.join(OBJ, name.replace(".hip", ".o"))
    cmd = ["hipcc", "-c", src, "-o", obj] + COMMON + extra
    if name in HAND_PLACED:
        cmd.append("-save-temps=obj")   # keeps the device assembly beside the object, for the check below
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass warns that it does not know the packed-fp32 feature; that is expected
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {name}:\n{err}")
    if err.strip() and verbose:
        print(err, flush=True)
    if name in HAND_PLACED:
        asm = os.path.join(OBJ, name.replace(".hip", "-hip-amdgcn-amd-amdhsa-gfx950.s"))
        check_accumulation_registers(asm)
        check_pending_reads(asm)
        check_matrix_operands(asm)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=6) as ex:
        objs = list(ex.map(lambda kv: _compile(kv[0], kv[1], verbose), SOURCES.items()))
    cmd = ["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-o", OUT] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
