"""Builds ``libtictac.so`` from ``csrc/`` with hipcc for gfx950 (cross-compiles without a GPU), and ``_layers.so``, the compiled
half of ``layers.py``, with the host compiler."""

from __future__ import annotations

import glob
import os
import re
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtictac.so")
LAYERS = os.path.join(HERE, "_layers.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def is_stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(LAYERS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(LAYERS))
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(f) > t for f in deps)


# Kernels whose waits for memory are counted by hand ("s_waitcnt vmcnt(N)" in inline asm): the count is right only
# while the compiler issues exactly the memory instructions the source shows between two such waits.  For each
# kernel (by a piece of its mangled name): N, and what must lie between consecutive hand-written waits.
#   "level": exactly `loads` 16-byte loads and `stores` stores, nothing else that counts (N = 7 levels of them)
#   "request": after the stores that follow a wait come `loads` 16-byte loads in straight-line code (the request
#              the wait is counted for); up to the next wait only loads follow (a load whose value is used has
#              been waited for, and everything older with it: memory instructions of a wave complete in order)
#   "stores": in the loops of the waves that store, N = 6 k: k 16-byte stores and no other memory instruction between the wait and
#             the branch, barrier or wait before it (a loop stores k rows per level; all of k = 1 .. n occur)
COUNTED_WAITS = {
    "16propagate_levelsILi": {"n": 21, "kind": "level", "loads": 2, "stores": 1},
    "22propagate_levels_batchILi": {"n": 21, "kind": "level", "loads": 2, "stores": 1},
    "24propagate_levels_q_batchILi": {"n": 14, "kind": "level", "loads": 1, "stores": 1},
    "15propagate_nodesILi": {"n": 8, "kind": "request", "loads": 8},
    "25propagate_levels_q_storedILi": {"n": 7, "kind": "stores"},
}
_VM_PREFIXES = ("global_", "flat_", "scratch_", "buffer_")


def _functions(asm: str):
    """(name, lines) of every function in the assembly text."""
    name, lines = None, []
    for line in asm.splitlines():
        head = line.split(";")[0].rstrip()
        if head.startswith("_Z") and head.endswith(":"):
            name, lines = head[:-1], []
            continue
        if name is None:
            continue
        lines.append(line)
        if line.strip().startswith(".Lfunc_end"):
            yield name, lines
            name = None


def check_counted_waits(asm: str) -> list:
    """Violations (strings) of the rules above in the device assembly of k1_propagate.hip; [] when it is sound."""
    bad, seen = [], set()
    for name, lines in _functions(asm):
        rule = next((r for key, r in COUNTED_WAITS.items() if key in name), None)
        if rule is None:
            continue
        seen.add(next(key for key in COUNTED_WAITS if key in name))
        in_asm, events = False, []          # ("wait", n) | ("vm", mnemonic) | ("branch",)
        for line in lines:
            t = line.strip()
            if t.startswith(";;#ASMSTART"):
                in_asm = True
            elif t.startswith(";;#ASMEND"):
                in_asm = False
            elif t.startswith("s_waitcnt") and in_asm and "vmcnt(" in t:
                n = int(t.split("vmcnt(")[1].split(")")[0])
                if n > 0:
                    events.append(("wait", n))
            elif t.startswith(_VM_PREFIXES):
                events.append(("vm", t.split()[0]))
            elif t.startswith(("s_cbranch", "s_branch", "s_swappc", "s_setpc", "s_barrier")):
                events.append(("branch",))
        spills = ("scratch_",) if rule["kind"] == "stores" else ("scratch_", "buffer_")
        if any(e[0] == "vm" and e[1].startswith(spills) for e in events):
            bad.append(f"{name}: register spills (scratch instructions) in a kernel with counted waits")
        waits = [i for i, e in enumerate(events) if e[0] == "wait"]
        if not waits:
            bad.append(f"{name}: no hand-written wait found")
            continue
        if rule["kind"] == "stores":
            found = set()
            for i in waits:
                first = i
                while first > 0 and events[first - 1][0] == "vm":
                    first -= 1
                ops, n = [e[1] for e in events[first:i]], events[i][1]
                if n % 6 or len(ops) != n // 6 or any(o != "buffer_store_dwordx4" for o in ops):
                    bad.append(f"{name}: {ops} before a wait for all but {n}")
                found.add(n // 6)
            if found != set(range(1, rule["n"] + 1)):
                bad.append(f"{name}: loops that store {sorted(found)} rows per level, expected 1 to {rule['n']}")
            continue
        if any(events[i][1] != rule["n"] for i in waits):
            bad.append(f"{name}: a hand-written wait is not vmcnt({rule['n']})")
        if rule["kind"] == "level":
            for a, b in zip(waits, waits[1:]):
                ops = [e[1] for e in events[a + 1:b] if e[0] == "vm"]
                loads = sum(o == "global_load_dwordx4" for o in ops)
                stores = sum(o.startswith("global_store") for o in ops)
                if loads != rule["loads"] or stores != rule["stores"] or len(ops) != loads + stores:
                    bad.append(f"{name}: {ops} between two waits, expected {rule['loads']} loads and "
                               f"{rule['stores']} stores")
                    break
        else:
            for k, a in enumerate(waits):
                b = waits[k + 1] if k + 1 < len(waits) else len(events)
                region = events[a + 1:b]
                stores = [i for i, e in enumerate(region) if e[0] == "vm" and e[1].startswith("global_store")]
                first = (stores[-1] + 1) if stores else 0
                while first < len(region) and region[first][0] != "vm":
                    first += 1
                request = region[first:first + rule["loads"]]
                ok = len(request) == rule["loads"] and all(e == ("vm", "global_load_dwordx4") for e in request)
                ok = ok and all("load" in e[1] for e in region[first + rule["loads"]:] if e[0] == "vm")
                if not ok:
                    bad.append(f"{name}: after a wait, the stores are not followed by {rule['loads']} straight-line "
                               f"16-byte loads and then loads only")
                    break
    for key in COUNTED_WAITS:
        if key not in seen:
            bad.append(f"no kernel matching {key} in the assembly")
    return bad


# The matrix instructions of these kernels are written in asm, in place, so that their accumulators stay where they are; the compiler does not know
# how long their results take, so it must not move an accumulator beside them, and that they need what a vector instruction wrote two instructions earlier.
ACCUMULATORS = "18product_kernel_256"
ACCUMULATORS_F8 = ("21product_f8_kernel_256", "17product_f8_kernelI")


def _registers(operands: str) -> set:
    """The vector and accumulation registers that a list of operands names."""
    found = set()
    for kind, first, last, one in re.findall(r"\b([av])(?:\[(\d+):(\d+)\]|(\d+))", operands):
        found.update((kind, n) for n in range(int(first or one), int(last or one) + 1))
    return found


def check_accumulators(asm: str, kernel: str = ACCUMULATORS) -> list:
    """Violations (strings) in the device assembly of a source of products: an accumulator read, written or moved in a stretch of code without labels
    that holds matrix instructions, or read before the wait that follows them, and registers that spill; [] when it is sound."""
    bad, seen = [], 0
    for name, lines in _functions(asm):
        if kernel not in name:
            continue
        seen += 1
        multiplies = moves = waited = spilled = early = mixed = 0
        for line in lines + [".end:"]:
            t = line.strip()
            if t.startswith(".") and t.split()[0].endswith(":"):
                mixed += bool(multiplies and moves)
                multiplies = moves = 0
            elif t.startswith("v_mfma"):
                multiplies += 1
                waited = 0
            elif t.startswith("s_nop 15"):
                waited = 1
            elif t.startswith("v_accvgpr"):
                moves += 1
                early += t.startswith("v_accvgpr_read") and not waited
            elif t.startswith(("ds_write", "global_store")) and any(kind == "a" for kind, _ in _registers(t.split(";")[0])):
                moves += 1
                early += not waited
            elif t.startswith("scratch_"):
                spilled += 1
        if mixed:
            bad.append(f"{name}: accumulators are moved among the matrix instructions")
        if early:
            bad.append(f"{name}: accumulators are read before the wait")
        if spilled:
            bad.append(f"{name}: register spills (scratch instructions)")
    if not seen:
        bad.append(f"no kernel {kernel} found")
    return bad


def check_operands(asm: str, kernel: str) -> list:
    """Violations (strings) in the device assembly of a source of products: a matrix instruction that reads a register which one of the two instructions
    before it wrote, along the text and along every branch (an "s_nop N" counts N + 1); [] when it is sound."""
    bad = []
    for name, lines in _functions(asm):
        if kernel not in name:
            continue
        code, at = [], {}                       # (mnemonic, operands); label: the instruction behind it
        for line in lines:
            t = line.split(";")[0].strip()
            if t.startswith(".") and t.split()[0].endswith(":"):
                at[t.split()[0][:-1]] = len(code)
            elif t and not t.startswith("."):
                op, _, rest = t.partition(" ")
                code.append((op, rest.strip()))

        def written(i):
            op, rest = code[i]
            return _registers(rest.split(",")[0]) if op.startswith("v_") and not op.startswith(("v_mfma", "v_cmp")) else set()

        def short(i, reads, waits, came):
            """whether, going back from in front of instruction i, one of `reads` was written less than `waits` instructions ago"""
            while waits > 0:
                for j in came.get(i, ()):
                    if short(j + 1, reads, waits, {}):
                        return True
                i -= 1
                if i < 0 or code[i][0] in ("s_branch", "s_endpgm", "s_setpc_b64"):
                    return False
                if written(i) & reads:
                    return True
                waits -= int(code[i][1]) + 1 if code[i][0] == "s_nop" else 1
            return False

        came = {}
        for j, (op, rest) in enumerate(code):
            if op.startswith(("s_cbranch", "s_branch")) and rest in at:
                came.setdefault(at[rest], []).append(j)
        for i, (op, rest) in enumerate(code):
            if op.startswith("v_mfma") and short(i, _registers(rest.split(",", 1)[1]), 2, came):
                bad.append(f"{name}: {op} {rest} reads what was written right before it")
    return bad


def check_products_f8(asm: str) -> list:
    return [x for kernel in ACCUMULATORS_F8 for check in (check_accumulators, check_operands) for x in check(asm, kernel)]


def device_assembly(source: str) -> str:
    cmd = [HIPCC] + [f for f in FLAGS if f not in ("-shared", "-fPIC")] + \
        ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S", "-o", "-", source]
    return subprocess.run(cmd, check=True, stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True).stdout


def build_layers(verbose: bool = False) -> str:
    import sysconfig
    import torch
    root, rocm = os.path.dirname(torch.__file__), os.path.dirname(os.path.dirname(HIPCC))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
               os.path.join(rocm, "include"), os.path.join(ROOT, "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] + [f"-I{d}" for d in include] + \
        ["-o", LAYERS, os.path.join(CSRC, "layers_binding.cpp"), "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_hip", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return LAYERS


CHECKS = {"k1_propagate.hip": check_counted_waits, "k8_product.hip": check_accumulators, "k9_product.hip": check_products_f8}


def build(verbose: bool = False) -> str:
    compile_flags = [f for f in FLAGS if f != "-shared"] + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as jobs:
        def compiled(source):
            to = os.path.join(objects, os.path.basename(source) + ".o")
            cmd = [HIPCC] + compile_flags + ["-c", "-o", to, source]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.check_call(cmd)
            return to

        checks = {name: jobs.submit(lambda name, check: check(device_assembly(os.path.join(CSRC, name))), name, check) for name, check in CHECKS.items()}
        found = list(jobs.map(compiled, sorted(sources(), key=os.path.getsize, reverse=True)))
        for source, check in checks.items():
            if check.result():
                if os.path.exists(LIB):
                    os.remove(LIB)
                raise RuntimeError(f"{source}: what is written by hand no longer matches the generated code:\n  " + "\n  ".join(check.result()))
        subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + sorted(found))
    build_layers(verbose)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    print(LIB)
