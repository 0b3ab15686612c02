"""Kernels that bring memory straight into LDS and wait for a number of requests, counted by hand: the code that was built has at least as many behind
those that are waited for.  (A request that the compiler drops, merges with another or moves in front would make such a wait too short.)"""
import os
import re
import struct
import subprocess

import pytest

import paper_1512_02595_amd
from paper_1512_02595_amd import build

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin", "llvm-objdump")


def amdgpu_objects(data):
    at = data.find(b"\x7fELF", 1)
    while at >= 0:
        if struct.unpack_from("<H", data, at + 18)[0] == 224:                    # EM_AMDGPU
            sections = struct.unpack_from("<Q", data, at + 40)[0]
            size, count = struct.unpack_from("<HH", data, at + 58)
            yield data[at:at + sections + size * count]
        at = data.find(b"\x7fELF", at + 1)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Instructions of the kernels in question, by their names."""
    folder, found = tmp_path_factory.mktemp("code"), {}
    with open(os.path.join(os.path.dirname(paper_1512_02595_amd.__file__), "libctc_mi355x.so"), "rb") as f:
        data = f.read()
    for code in amdgpu_objects(data):
        names = {n.decode() for n in re.findall(rb"_ZN5layer[A-Za-z0-9_]*(?:linear_tiles|gradient_wide)_kernel[A-Za-z0-9_]*", code)}
        names = sorted(n for n in names if not n.endswith(".kd"))
        if not names:
            continue
        (folder / "code.o").write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--disassemble-symbols=" + ",".join(names), str(folder / "code.o")],
                              check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"<(_ZN5layer\w+)>:\n(.*?)(?=\n\n|\Z)", text, flags=re.S):
            found[name] = [line.split("//")[0].strip() for line in body.split("\n")]
    return found


def requests_behind(code, wait):
    """For each of the waits: what is asked of memory from it to the next branch, wait of its kind or end, in order."""
    out = []
    for i, line in enumerate(code):
        if not re.search(wait, line):
            continue
        asked = []
        for later in code[i + 1:]:
            if re.match(r"s_c?branch|s_endpgm", later) or re.search(wait, later):
                break
            if re.match(r"(global|buffer|flat|scratch)_(load|store|atomic)", later):
                asked.append(later.split()[0])
        out.append(asked)
    return out


def test_the_kernels_are_there(kernels):
    assert sum("linear_tiles" in n for n in kernels) == 8 and sum("gradient_wide" in n for n in kernels) == 2


def test_weights_gradient_in_wide_tiles(kernels):
    """Numbers for the step behind are asked for four requests at a time, first of a step's fourteen; the wait of the step in between and its own leave 24."""
    for name in (n for n in kernels if "gradient_wide" in n):
        behind = requests_behind(kernels[name], r"s_waitcnt vmcnt\(24\)")
        assert len(behind) == 3, name
        for asked in behind:
            assert len(asked) == 14, (name, asked)
            assert all("lds" in a for a in asked[:4]) and not any("lds" in a for a in asked[4:]), (name, asked)


def test_activations_in_tiles(kernels):
    """A step asks for its tile's rows and symbols, a request each for 64 of them; two steps' requests stay under way."""
    for name in (n for n in kernels if "linear_tiles" in n):
        each = sum(map(int, re.search(r"Li(\d)ELi(\d)E", name).groups()))
        code = kernels[name]
        behind = requests_behind(code, rf"s_waitcnt vmcnt\({2 * each}\)")
        assert len(behind) == 7, (name, len(behind))      # four steps of the loop, up to three behind it
        for asked in behind:                              # (behind the last step come the loads of what is written)
            assert len([a for a in asked if "lds" in a]) == each and all("lds" in a for a in asked[:each]), (name, asked)
        first = next(i for i, line in enumerate(code) if re.search(rf"s_waitcnt vmcnt\({3 * each}\)", line))
        before = [line for line in code[:first] if "_load_lds_" in line]
        assert len(before) == 4 * each, name
