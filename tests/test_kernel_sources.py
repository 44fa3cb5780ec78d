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


def test_assembly_names_the_special_registers_that_it_writes():
    """m0, vcc, exec and scc are the compiler's too: what an instruction's first operand writes has to be among the clobbers."""
    found, wrote = 0, 0
    for path, text in statements():
        found += 1
        strings = re.findall(r'"((?:[^"\\]|\\.)*)"', text)
        for reg in ("m0", "vcc", "exec", "scc"):
            if re.search(rf"(?:^|\\n|\\t|;)\s*[sv]_\w+ {reg}\b", strings[0]):
                wrote += 1
                assert reg in strings[1:], f"{path}: {text}"
    assert found > 10 and wrote >= 2
