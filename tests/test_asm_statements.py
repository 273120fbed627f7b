"""Assembly statements of the kernels name the registers that they write (CPU only)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_10071_amd", "csrc")


def statements():
    """(file, code, clobbers) of every asm statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        src = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", src):
            depth, end = 1, m.end()
            quoted = False
            while depth:
                c = src[end]
                if c == '"' and src[end - 1] != "\\":
                    quoted = not quoted
                elif not quoted:
                    depth += (c == "(") - (c == ")")
                end += 1
            body = src[m.end():end - 1]
            # code : outputs : inputs : clobbers, with the colons outside quotes
            parts, inside = [""], False
            for c in body:
                inside ^= c == '"'
                if c == ":" and not inside:
                    parts.append("")
                else:
                    parts[-1] += c
            yield os.path.basename(path), parts[0], parts[3] if len(parts) > 3 else ""


def test_m0_is_named_where_it_is_written():
    found = list(statements())
    assert len(found) > 5
    writes = [s for s in found if re.search(r"\bs_\w+\s+m0\s*,", s[1])]
    assert writes
    for name, code, clobbers in writes:
        assert '"m0"' in clobbers, (name, code)
