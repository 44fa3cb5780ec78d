"""Rules that the kernel sources keep and no run of them shows."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_28458_amd", "csrc")


def statements():
    """Every inline assembly statement, to its semicolon outside of strings."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        text = open(path).read()
        for m in re.finditer(r'\basm\b(?:\s+volatile)?\s*\((?:[^";]|"(?:[^"\\]|\\.)*")*;', text):
            yield os.path.basename(path), m.group(0)


def test_assembly_leaves_the_special_registers_as_they_were():
    """m0, vcc, exec and scc are the compiler's too.  vcc and scc may be named as clobbers; m0 and exec are reserved, which
    clobbers do not cover: what writes them saves them first and puts them back at its end."""
    found, wrote = 0, 0
    for path, text in statements():
        found += 1
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', text)
        lines = [x.strip() for x in re.split(r"(?:\\n|\\t|;)+", strings[0]) if x.strip()]
        for reg in ("m0", "vcc", "exec", "scc"):
            if any(re.match(rf"[sv]_\w+ {reg}\b", x) for x in lines):
                wrote += 1
                saved = re.fullmatch(rf"s_mov_b(?:32|64) (%\d), {reg}", lines[0])
                restored = saved and re.fullmatch(rf"s_mov_b(?:32|64) {reg}, {saved.group(1)}", lines[-1])
                assert restored or reg in ("vcc", "scc") and reg in strings[1:], f"{path}: {text}"
    assert found > 10 and wrote >= 2
