"""What the compiler is told about LDS that one wave's lanes hand each other, read from the device code's IR (no GPU)."""
import os
import re
import subprocess

from paper_2609_36835_amd import build as B


def kernels_ir(source, tmp_path):
    """{mangled name: [basic blocks' lines]} of a source's kernels."""
    out = os.path.join(tmp_path, "device.ll")
    cmd = [B._hipcc(), *B.COMMON_FLAGS, "-x", "hip", "--cuda-device-only", "-emit-llvm", "-S",
           os.path.join(B.CSRC, source), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    with open(out) as f:
        text = f.read()
    found = {}
    for m in re.finditer(r"^define [^\n]*amdgpu_kernel void @(\w+)\(.*?^}", text, re.M | re.S):
        found[m[1]] = [b.split("\n") for b in re.split(r"\n(?=[\w.]+:)", m[0])]
    return found


def exchanges(lines, kind):
    """A basic block's LDS stores (w) and loads (r) of the types `kind` matches, and its fences (f), in order."""
    s = ""
    for line in lines:
        if re.search(rf"store {kind} .*ptr addrspace\(3\)", line):
            s += "w"
        elif re.search(rf"load {kind}, ptr addrspace\(3\)", line):
            s += "r"
        elif re.search(r"\bfence\b", line):
            s += "f"
    return s


def test_attention_keys_are_fenced_on_both_sides(tmp_path):
    """A wave's keys go through LDS to other lanes in every turn of the loop over blocks: stores, a fence, loads, and a
    fence again before the next turn's stores, with a bias and without."""
    found = {n: b for n, b in kernels_ir("attend_q.hip", tmp_path).items() if "k_attendq_partial" in n}
    loops = 0
    for name, blocks in found.items():
        for lines in blocks:
            s = exchanges(lines, r"<(?:4 x i32|16 x i8)>")
            if "w" not in s:
                continue
            loops += 1
            assert "r" in s, name                    # the loop's body is one block: its end meets its beginning
            twice = s + s
            assert not re.search("wr|rw", twice), (name, s)
    assert len(found) == 36 and loops == 24, (len(found), loops)   # the 16-wave kernels keep their keys in registers
