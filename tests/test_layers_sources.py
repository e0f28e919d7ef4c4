"""What inline assembly reads and writes is declared to the compiler: loads into LDS
take their LDS address from m0, which is an operand of theirs."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def statements():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2608_15438_amd", "csrc", "*"))):
        with open(path) as f:
            for m in re.finditer(r"\basm\b[^;]*;", f.read()):
                yield os.path.basename(path), m.group(0)


def test_m0_is_an_operand():
    loads = 0
    for path, s in statements():
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(":", 1)[0]))
        assert not re.search(r"\bm0\b", code), (path, s)      # not written behind the compiler's back
        if "load_lds" in code:
            assert '"{m0}"(' in s, (path, s)
            loads += 1
    assert loads                                              # there are some
