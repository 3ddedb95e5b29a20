"""The loads through a buffer descriptor into LDS are written in inline asm too: in the built library each keeps the distances that
tests/test_load_lds_wait_states.py states, from the vector instruction that wrote a scalar register of its descriptor (5 wait states) and from
the scalar one that wrote m0 (1).  Reads the AMD assembly of the library built here."""
import os
import re
import subprocess

from tests.test_load_lds_wait_states import OBJDUMP, _code_objects, hazards


def _as_lds_load(line):
    """A buffer load into LDS as the rule's reader knows such loads: its offset and its descriptor."""
    m = re.match(r"\s*(?:buffer_load_dword\w*) (v\d+), (s\[\d+:\d+\]), 0 offen lds", line.split("//")[0])
    return f"global_load_lds_dwordx4 {m[1]}, {m[2]}" if m else line


def test_the_rule_on_buffer_loads():
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds // 0"
    early = ["0000 <k>:", "v_readfirstlane_b32 s6, v9", "s_mov_b32 m0, s3"]
    assert hazards([_as_lds_load(x) for x in early + [load]])[0]
    assert hazards([_as_lds_load(x) for x in early + ["s_nop 2", load]])[0]
    assert not hazards([_as_lds_load(x) for x in early + ["s_nop 4", load]])[0]
    assert hazards([_as_lds_load(x) for x in ["0000 <k>:", "s_add_u32 m0, m0, 0x400", load]])[0]
    assert not hazards([_as_lds_load(x) for x in ["0000 <k>:", "s_add_u32 m0, m0, 0x400", "s_nop 0", load]])[0]


def test_buffer_loads_into_lds_wait_for_their_descriptor(tmp_path):
    from paper_2512_16615_amd import build, llsa
    if not os.path.exists(llsa.LIB_PATH):
        build.build(verbose=False)
    found, loads = [], 0
    for i, code in enumerate(_code_objects(llsa.LIB_PATH)):
        obj = tmp_path / f"{i}.co"
        obj.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(obj)], check=True, capture_output=True, text=True).stdout
        lines = text.splitlines()
        turned = [_as_lds_load(x) for x in lines]
        loads += sum(a is not b for a, b in zip(lines, turned))
        assert not any(re.match(r"\s*buffer_load\S* .*\blds\b", x.split("//")[0]) for x in turned)      # every form of them is known
        found += hazards(turned)[0]
    assert loads > 100
    assert not found, f"{len(found)} of {loads} loads, the first: {found[0]}"
