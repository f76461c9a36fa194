"""The layer products load from memory straight into LDS in inline assembly, inside
which the compiler checks no hazards. This test disassembles the gfx950 code of
every unit of them and checks what makes those statements sound:

* the statement writes m0 from a scalar, then waits a state, then loads, with no
  branch into or out of the three; m0 appears nowhere else, and no other
  instruction reads it implicitly;
* a memory instruction needs five wait states after a vector instruction (a
  v_readfirstlane, the reload of a spilled scalar) writes a scalar of its
  descriptor;
* nothing is kept in scratch memory inside a loop with such loads: the loads in flight are
  counted, and a spill would be counted with them."""
import os
import re
import subprocess

import pytest

LLVM = "/opt/rocm/llvm/bin"
TARGET = "hipv4-amdgcn-amd-amdhsa--gfx950"
M0_READERS = re.compile(r"^(v_movrel|s_movrel|s_sendmsg|ds_gws|ds_append|ds_consume|v_interp|s_set_gpr_idx|"
                        r"global_load_lds)")


def _units():
    from paper_1909_10616_amd import build
    return [u[0] for u in build._units() if u[1] == "product_inst.hip"]


@pytest.fixture(scope="module")
def objects():
    from paper_1909_10616_amd import build
    paths = {u: os.path.join(build.BUILD, u + ".o") for u in _units()}
    if not all(os.path.exists(p) for p in paths.values()):
        build.build(incremental=True, verbose=False)
    return paths


def _kernels(obj, tmp_path):
    """Kernel → its instructions and the indexes that branches lead to."""
    fb, co = tmp_path / "fatbin", tmp_path / "device.co"
    subprocess.run([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fb}", obj], check=True)
    subprocess.run([f"{LLVM}/clang-offload-bundler", "--unbundle", "--type=o", f"--input={fb}",
                    f"--targets={TARGET}", f"--output={co}"], check=True)
    out, body, at, targets, start = {}, [], {}, set(), 0
    for line in subprocess.run([f"{LLVM}/llvm-objdump", "-d", str(co)], check=True,
                               capture_output=True, text=True).stdout.splitlines():
        m = re.match(r"^([0-9a-f]+) <(\w+)>:$", line)
        if m:
            start, body, at, targets = int(m.group(1), 16), [], {}, set()
            out[m.group(2)] = body, at, targets
        elif line.startswith("\t") and "//" in line:
            ins, _, note = line.partition("//")
            at[int(re.match(r"\s*([0-9A-F]+):", note).group(1), 16) - start] = len(body)
            body.append(ins.strip())
            if re.match(r"s_c?branch", body[-1]):
                targets.add(int(re.search(r"<\w+(?:\+0x([0-9a-f]+))?>", note).group(1) or "0", 16))
    return {k: (v, {at[t] for t in targets if t in at}) for k, (v, at, targets) in out.items()}


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m.group(1))} if m else set()


def _split(ins):
    op, _, rest = ins.partition(" ")
    return op, [a.strip() for a in rest.split(",")] if rest else []


@pytest.mark.parametrize("unit", _units())
def test_loads_into_lds_are_sound(objects, unit, tmp_path):
    kernels = _kernels(objects[unit], tmp_path)
    with_loads = 0
    for fn, (ins, targets) in kernels.items():
        inside, loads = set(), [i for i, x in enumerate(ins) if re.match(r"buffer_load\w* .*\blds\b", x)]
        with_loads += bool(loads)
        for at in loads:
            where = f"{unit} {fn}: {ins[max(at - 12, 0):at + 2]}"
            assert re.fullmatch(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds", ins[at]), where
            assert ins[at - 1] == "s_nop 0", where
            assert re.fullmatch(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi|0x[0-9a-f]+|\d+|ttmp\d+)", ins[at - 2]), where
            assert not targets & {at - 1, at}, where
            inside |= {at - 2, at}
            need, states = _scalars(_split(ins[at])[1][1]), 0
            assert len(need) == 4, where
            for before in reversed(ins[max(at - 10, 0):at]):
                if not need or states >= 5:
                    break
                op, args = _split(before)
                wrote = _scalars(args[0]) & need if args else set()
                assert not (wrote and op.startswith("v_")), where
                need -= wrote
                states += int(args[0], 0) + 1 if op == "s_nop" else 1
        for at, i in enumerate(ins):
            if at not in inside:
                assert not re.search(r"\bm0\b", i) and not M0_READERS.match(i), f"{unit} {fn}: {i}"
        if loads:
            span = [i for i in ins[loads[0]:loads[-1]] if i.startswith("scratch_")]
            assert not span, f"{unit} {fn}: {span[:4]}"
    assert with_loads >= 4   # (tiles and epilogues; the fewest in fp32 along k)
