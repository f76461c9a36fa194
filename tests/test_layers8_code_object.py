"""The 8-bit products load codes and scales from memory straight into LDS in inline assembly. On
the gfx950 code of every unit of them:

* either load stands right behind its write of m0 and one wait state, with no branch into
  or out of the three, and nothing else touches m0;
* five wait states lie between a vector instruction's write of a scalar and a load whose
  descriptor reads it;
* nothing is kept in scratch memory: the loads in flight are counted, and a spill would be
  counted with them;
* as many matrix instructions as a stage has: none was left out or made twice."""
import os
import re

import pytest

from test_layers_code_object import M0_READERS, _kernels, _scalars, _split


def _units():
    from paper_1909_10616_amd import build
    return [u[0] for u in build._units() if u[1] in ("product8_inst.hip", "rows8.hip")]


@pytest.fixture(scope="module")
def objects():
    from paper_1909_10616_amd import build
    paths = {u: os.path.join(build.BUILD, u + ".o") for u in _units()}
    if not all(os.path.exists(p) for p in paths.values()):
        build.build(incremental=True, verbose=False)
    return paths


LOAD = re.compile(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds|global_load_lds_dword v\[\d+:\d+\], off")
READERS = re.compile(M0_READERS.pattern.replace("|global_load_lds", ""))


@pytest.mark.parametrize("unit", _units())
def test_loads_into_lds_are_sound(objects, unit, tmp_path):
    kernels = {k: v for k, v in _kernels(objects[unit], tmp_path).items() if "product8_kernel" in k or "staged8" in k}
    assert len(kernels) == (40 if unit == "rows8" else 6 if unit.startswith("product8_0") else 11)
    for fn, (ins, targets) in kernels.items():
        loads = [i for i, x in enumerate(ins) if re.search(r"\blds\b", x) or "load_lds" in x]
        assert sum("global_load_lds" in ins[i] for i in loads) >= 2 and len(loads) > 8
        inside = set()
        for at in loads:
            where = f"{unit} {fn}: {ins[max(at - 12, 0):at + 2]}"
            assert LOAD.fullmatch(ins[at]), where
            assert ins[at - 1] == "s_nop 0", where
            assert re.fullmatch(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi|0x[0-9a-f]+|\d+|ttmp\d+)", ins[at - 2]), where
            assert not targets & {at - 1, at}, where
            inside |= {at - 2, at}
            if "buffer" not in ins[at]:
                continue
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
                assert not re.search(r"\bm0\b", i) and not READERS.match(i), f"{unit} {fn}: {i}"
        assert not [i for i in ins if i.startswith("scratch_")], f"{unit} {fn}"
        if unit == "rows8":
            continue
        exact = "ILi1ELb1E" in fn or "ILi0ELb1E" in fn
        stage = {"0": 32, "1": 16, "2": 8}[unit[9]] * (4 if exact else 1)
        assert sum("mfma" in i for i in ins) == stage, f"{unit} {fn}"
