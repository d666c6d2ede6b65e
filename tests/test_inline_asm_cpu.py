"""What the instructions in the sources say of themselves."""

import glob
import os
import re

import paper_2602_16994_amd as mpv


def statements():
    for path in sorted(glob.glob(os.path.join(os.path.dirname(mpv.lib_path()), "csrc", "*"))):
        with open(path) as f:
            for found in re.finditer(r'asm volatile\(((?:"(?:\\.|[^"])*"|[^";])*)\);', f.read()):
                yield os.path.basename(path), found.group(1)


def test_registers_that_an_instruction_writes_are_named():
    writes = 0
    for name, text in statements():
        code = "".join(re.findall(r'"((?:\\.|[^"])*)"', text.split("::")[0]))
        for instruction in code.split("\\n"):
            words = re.split(r"[\s,]+", instruction.replace("\\t", " ").strip())
            if len(words) > 1 and words[1] in ("m0", "vcc", "scc", "exec") and not words[0].startswith("s_cmp"):
                writes += 1
                assert f'"{words[1]}"' in text.split("::")[-1], (name, text)
    assert writes == 2
