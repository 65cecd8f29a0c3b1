"""Scalar registers that a vector instruction wrote are not read too early by a vector memory instruction: five wait states are between.  The compiler keeps
to that in its own code, not in the text of assembly statements."""
import os
import re
import shutil
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1912_08756_amd", "csrc")
LIBRARY = os.path.join(ROOT, "paper_1912_08756_amd", "libicq.so")
MEMORY = ("buffer_", "tbuffer_", "global_", "flat_", "scratch_")


def _states(line):
    """Wait states that an instruction stands for."""
    return int(line.split()[1], 0) + 1 if line.startswith("s_nop") else 1


# ---- the sources

def _statements():
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(\s*((?:\"(?:[^\"\\]|\\.)*\"\s*)+)(.*?)\);", text, flags=re.S):
            body = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m[1])).replace("\\t", " ").replace("\\n", "\n")
            yield name, [line.strip() for line in body.splitlines() if line.strip()], m[2]


def test_statements_with_memory_instructions_wait_for_their_scalar_operands():
    found = 0
    for name, lines, operands in _statements():
        scalar = '"s"' in operands
        for at, line in enumerate(lines):
            if scalar and line.startswith(MEMORY):
                found += 1
                assert sum(map(_states, lines[:at])) >= 5, (name, lines)
    assert found >= 2


# ---- the library as it is built

def _code_objects(path, folder):
    """The gfx950 code objects of a library: bundles begin with a magic word, then their entries' offsets, sizes and names."""
    data, magic, files, at = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", [], 0
    while (at := data.find(magic, at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count if count < 64 else 0):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            name = data[entry + 24:entry + 24 + length]
            if b"gfx950" in name and size > 0:
                files.append(os.path.join(str(folder), "%d.elf" % len(files)))
                with open(files[-1], "wb") as f:
                    f.write(data[at + offset:at + offset + size])
            entry += 24 + length
        at += 24
    return files


def _scalars(text):
    """Numbers of the scalar registers that operands name."""
    out = set()
    for first, last in re.findall(r"(?<![a-z0-9])s\[(\d+):(\d+)\]", text):
        out.update(range(int(first), int(last) + 1))
    out.update(map(int, re.findall(r"(?<![a-z0-9_\[:])s(\d+)\b", text)))
    return out


def _written(op, operands):
    """Scalar registers that a vector instruction writes."""
    if op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
        return _scalars(operands.split(", ")[0])
    return _scalars(operands.split(", ")[1]) if re.match(r"v_(add|sub|subrev|addc|subb|subbrev)_co_|v_div_scale|v_mad_[iu]64", op) else set()


def _too_early(lines):
    """(function, writer, reader, wait states between them) of every place that keeps too little distance."""
    found, function, written, now = [], "", [], 0              # written: (time, registers, line) of the last few
    for line in lines:
        if line.endswith(">:\n"):
            function, written = line.split("<")[1][:-3], []
            continue
        line = line.split("//")[0].strip()
        if not line or line[0] not in "bgfstv":
            continue
        op, _, operands = line.partition(" ")
        if op in ("s_branch", "s_endpgm", "s_setpc_b64"):      # (what follows is reached from elsewhere)
            written = []
        if written and op.startswith(MEMORY):
            reads = _scalars(operands)
            found += [(function, writer, line, now - when) for when, registers, writer in written if registers & reads and now - when < 5]
        now += _states(line)
        if op.startswith("v_"):
            registers = _written(op, operands)
            if registers:
                written.append((now, registers, line))
        if written and now - written[0][0] >= 5:
            written = [w for w in written if now - w[0] < 5]
    return found


def test_the_reading_of_listings():
    """What is too early, and what is not, in listings by hand."""
    def places(*lines):
        return [found[3] for found in _too_early(["0 <f>:\n"] + ["\t%s  // 0: 0\n" % line for line in lines])]

    load, m0 = "buffer_load_dwordx4 v1, s[4:7], s9 offen lds", "s_mov_b32 m0, s3"
    assert places("v_readlane_b32 s9, v198, 7", m0, "s_nop 0", load) == [2]
    assert places("v_readlane_b32 s9, v198, 7", m0, "s_nop 3", load) == []
    assert places("v_readfirstlane_b32 s4, v1", m0, "s_nop 2", load) == [4]
    assert places("v_readfirstlane_b32 s8, v1", m0, "s_nop 0", load) == []
    assert places("v_cmp_gt_f32_e64 s[8:9], v1, v2", "v_add_u32_e32 v1, s8, v2", load) == [1]
    assert places("v_mad_u64_u32 v[2:3], s[10:11], v5, s9, v[2:3]", load) == []
    assert places("v_readlane_b32 s9, v198, 7", "s_branch 12", load) == []


def test_the_built_library_keeps_the_distance(tmp_path):
    tool = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
    if not os.path.exists(LIBRARY) or not os.path.exists(tool):
        pytest.skip("needs the built library and llvm-objdump")
    files = _code_objects(LIBRARY, tmp_path)
    assert files
    memory = 0
    for path in files:
        with subprocess.Popen([tool, "-d", "--no-show-raw-insn", path], stdout=subprocess.PIPE, text=True) as listing:
            lines = listing.stdout.readlines()
        assert listing.returncode == 0
        memory += sum("buffer_load" in line for line in lines)
        found = _too_early(lines)
        assert not found, (len(found), found[:3])
    assert memory > 0
