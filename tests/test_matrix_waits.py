"""Between a matrix instruction and the first use of its result by anything but a matrix instruction that adds to it, the hardware asks for a number of
other instructions (it does not wait by itself).  The compiler counts them, and has once counted too few where a branch lay between: a result was read
half finished.  So: in every kernel of the delta rule, on every path, at least as many as the least that it leaves where no branch lies between, for the
same instruction.  Read from the library as built (no GPU needed)."""
import os
import re
import subprocess
from collections import defaultdict

import pytest

from paper_1901_10997_amd import build

LLVM = "/opt/rocm/llvm/bin"
TARGET = "hipv4-amdgcn-amd-amdhsa--gfx950"
TOOLS = ("llvm-objcopy", "clang-offload-bundler", "llvm-objdump")
FAR = 24            # more than any instruction asks for


def registers(text):
    out = set()
    for m in re.finditer(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))(?![\w\]])", text):
        lo, hi = (int(m[2]), int(m[3])) if m[2] else (int(m[4]), int(m[4]))
        out |= {(m[1], k) for k in range(lo, hi + 1)}
    return out


def kernels(text):
    """name -> [(address, instruction, address it may branch to)]"""
    found = {}
    for part in re.split(r"^(?=[0-9a-f]{16} <)", text, flags=re.M)[1:]:
        head, _, body = part.partition("\n")
        start, name = re.match(r"([0-9a-f]{16}) <(\S+)>:", head).groups()
        found[name] = []
        for line in body.split("\n"):
            m = re.match(r"\t(\S.*?)\s*// ([0-9A-F]{12}): [0-9A-F ]+(?:<\S+?\+0x([0-9a-f]+)>)?", line)
            if m:
                to = int(start, 16) + int(m[3], 16) if m[3] else None
                found[name].append((int(m[2], 16), m[1], to))
    return found


def distances(code):
    """(instruction, how its result is used) -> least number of instructions between, without a branch between and with one"""
    at = {address: i for i, (address, _, _) in enumerate(code)}
    follow = []
    for i, (_, text, to) in enumerate(code):
        op = text.split()[0]
        branches = op == "s_branch" or op.startswith("s_cbranch")
        nexts = [] if op in ("s_branch", "s_endpgm") or i + 1 == len(code) else [(i + 1, False)]
        if branches and to in at:
            nexts.append((at[to], True))
        follow.append([(j, took or branches) for j, took in nexts])
    least = defaultdict(lambda: [FAR, FAR])
    for i, (_, text, _) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        result, seen, stack = registers(text.split(",")[0]), {}, [(j, 0, branch) for j, branch in follow[i]]
        while stack:
            j, far, branch = stack.pop()
            if far > FAR or seen.get((j, branch), FAR + 1) <= far:
                continue
            seen[j, branch] = far
            use = code[j][1]
            op, _, args = use.partition(" ")
            kind = None
            if op.startswith("v_mfma"):
                parts = args.split(",")
                if (registers(parts[1]) | registers(parts[2])) & result:
                    kind = "operand"
                elif registers(parts[0]) & result:
                    continue        # adds to it, or starts another result in its place
            elif not op.startswith("s_") and registers(args) & result:
                kind = "other"
            if kind:
                slot = least[text.split()[0], kind]
                slot[branch] = min(slot[branch], far)
                continue
            step = int(args, 0) + 1 if op == "s_nop" else 1
            stack += [(n, far + step, branch or b) for n, b in follow[j]]
    return least


def library(tmp):
    if not os.path.exists(build.LIB):
        build.build()
    fat = os.path.join(tmp, "fat")
    subprocess.run([f"{LLVM}/llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", build.LIB, os.path.join(tmp, "unused")], check=True)
    data = open(fat, "rb").read()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__|CCOB", data)] + [len(data)]
    for a, b in zip(starts, starts[1:]):
        bundle, obj = os.path.join(tmp, "bundle"), os.path.join(tmp, "object")
        with open(bundle, "wb") as f:
            f.write(data[a:b])
        subprocess.run([f"{LLVM}/clang-offload-bundler", "--type=o", "--unbundle", f"--input={bundle}", f"--targets={TARGET}", f"--output={obj}"], check=True)
        names = subprocess.run([f"{LLVM}/llvm-objdump", "-t", obj], check=True, capture_output=True, text=True).stdout
        if "delta_walk_kernel" in names:
            yield subprocess.run([f"{LLVM}/llvm-objdump", "-d", obj], check=True, capture_output=True, text=True).stdout


@pytest.mark.skipif(not all(os.path.exists(f"{LLVM}/{t}") for t in TOOLS), reason="no LLVM tools")
def test_no_result_is_used_before_it_is_there(tmp_path):
    checked, least = 0, {}
    for text in library(str(tmp_path)):
        for name, code in kernels(text).items():
            if any(i.startswith("v_mfma") for _, i, _ in code):
                least[name] = distances(code)
                checked += 1
    assert checked >= 50
    straight = defaultdict(lambda: FAR)
    for found in least.values():
        for key, (without, _) in found.items():
            straight[key] = min(straight[key], without)
    assert 0 < straight["v_mfma_f32_16x16x32_bf16", "other"] < FAR
    short = {(name, key): (branch, straight[key]) for name, found in least.items() for key, (_, branch) in found.items() if branch < straight[key]}
    assert not short


def test_the_count_sees_what_it_looks_for():
    """A branch whose target reads the result at once, and the same with a wait in front."""
    def code(waits):
        lines = ["v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]", "s_cbranch_scc1 2", "s_nop 7", "s_nop 7"] + waits + ["v_accvgpr_read_b32 v9, a3", "s_endpgm"]
        return [(4 * i, line, 16 if line.startswith("s_cbranch") else None) for i, line in enumerate(lines)]

    key = ("v_mfma_f32_16x16x32_bf16", "other")
    assert distances(code([]))[key] == [FAR, 1]
    assert distances(code(["s_nop 6"]))[key] == [FAR, 8]
