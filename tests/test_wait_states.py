"""Wait states in the built library's gfx950 code (no GPU).

Two rules of this target that the hardware does not keep by itself, and that the
compiler does not keep inside a string of inline assembly:
  - a load into LDS takes its place there from M0; a scalar instruction that writes M0
    has to be one wait state at least before it (one instruction between the two);
  - a scalar register that a vector instruction wrote has to be five wait states old
    before a memory instruction of the vector unit takes its address from it.
Every instruction between the two counts as one, ``s_nop n`` as n + 1.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_30310_amd.build import LIB_PATH

OBJDUMP = shutil.which("llvm-objdump", path=os.pathsep.join(["/opt/rocm/llvm/bin", os.environ.get("PATH", "")]))
MEMORY = ("global_", "buffer_", "scratch_", "flat_")
SCALAR = re.compile(r"s\[(\d+):(\d+)\]|\bs(\d+)\b|\b(vcc)\b")


def scalars(text):
    """The scalar registers that operands name; VCC by its name."""
    regs = set()
    for lo, hi, one, vcc in SCALAR.findall(text):
        regs |= set(range(int(lo), int(hi) + 1)) if lo else {int(one)} if one else {vcc}
    return regs


def vector_writes(op, args):
    """The scalar registers that a vector instruction writes: lane reads, compares and carries."""
    if op.startswith(("v_readlane", "v_readfirstlane")):
        return scalars(args[0])
    if op.startswith("v_cmp_"):
        return scalars(args[0])
    if "_co_" in op or op.startswith(("v_div_scale", "v_mad_u64_u32", "v_mad_i64_i32")):
        return scalars(args[1])
    return set()


def breaches(listing):
    """The instructions of a listing that come too early, and what they wait for."""
    found, written, m0_age, name = [], {}, None, ""   # written: register -> wait states since a vector instruction wrote it
    for line in listing:
        line = line.split("//")[0].strip()
        if line.endswith(">:"):
            name = line
        if not line or line.endswith(":") or not re.match(r"[a-z]+_[a-z0-9_]+(\s|$)", line):
            continue
        op, _, rest = line.partition(" ")
        args = [a.strip() for a in rest.split(",")]
        if op.startswith(MEMORY):
            if re.search(r"\blds\b", rest) or "_lds_" in op:
                if m0_age == 0:
                    found.append((name, line, "M0"))
            for r in scalars(rest):
                if written.get(r, 5) < 5:
                    found.append((name, line, r))
        age = int(rest) + 1 if op == "s_nop" else 1
        written = {r: n + age for r, n in written.items() if n + age < 5}
        m0_age = None if m0_age is None else m0_age + age
        if op.startswith("v_"):
            for r in vector_writes(op, args):
                written[r] = 0
        elif op.startswith("s_") and args[0]:
            if args[0] == "m0":
                m0_age = 0
            for r in scalars(args[0]):   # a scalar instruction's result is seen at once
                written.pop(r, None)
    return found


def test_the_rules_on_short_listings():
    lines = lambda text: text.strip().splitlines()
    assert breaches(lines("s_mov_b32 m0, s2\nglobal_load_lds_dwordx4 v[0:1], off"))
    assert breaches(lines("s_add_u32 m0, s2, 4\nbuffer_load_dwordx4 v1, s[4:7], 0 offen lds"))
    assert not breaches(lines("s_mov_b32 m0, s2\ns_nop 0\nglobal_load_lds_dword v[0:1], off"))
    assert not breaches(lines("s_mov_b32 m0, s2\nglobal_load_dword v1, v[0:1], off"))
    late = "v_readlane_b32 s62, v4, 0\n%s\nglobal_load_lds_dwordx4 v10, s[62:63]"
    assert breaches(lines(late % "s_nop 3")) and not breaches(lines(late % "s_nop 4"))
    assert breaches(lines(late % "v_mov_b32_e32 v1, v2\ns_nop 2"))
    assert not breaches(lines("v_readlane_b32 s62, v4, 0\ns_mov_b64 s[8:9], s[62:63]\nglobal_load_dword v1, v0, s[8:9]"))
    assert not breaches(lines("v_readlane_b32 s62, v4, 0\ns_mov_b32 s62, s1\nglobal_load_dword v1, v0, s[62:63]"))
    assert breaches(lines("v_cmp_lt_u32_e64 s[2:3], v0, v1\nbuffer_load_dword v1, v0, s[0:3], 0 offen"))
    assert breaches(lines("v_add_co_u32_e64 v0, s[2:3], v0, v1\nglobal_store_dword v1, v0, s[2:3]"))


@pytest.mark.skipif(OBJDUMP is None, reason="no disassembler")
def test_the_library_waits(tmp_path):
    shutil.copy(LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(p for p in os.listdir(tmp_path) if p.endswith("gfx950"))
    assert objects
    found, loads = [], 0
    for o in objects:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", o], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        loads += text.count("global_load_lds_")
        found += breaches(text.splitlines())
    assert loads > 100   # (the listings are what they are taken for)
    print("\n".join(map(str, found[:20])))
    assert not found, f"{len(found)} instructions come too early"
