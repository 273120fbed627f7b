"""Assembly statements of the kernels leave to the compiler what it has to know (CPU only)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_10071_amd", "csrc")


def statements():
    """(file, code, inputs) of every asm statement."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        src = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\s+(?:volatile\s*)?\(", src):
            # code : outputs : inputs : clobbers, with the colons outside quotes
            parts, quoted, depth = [""], False, 1
            for c in src[m.end():]:
                quoted ^= c == '"'
                depth += 0 if quoted else (c == "(") - (c == ")")
                if not depth:
                    break
                if c == ":" and not quoted:
                    parts.append("")
                else:
                    parts[-1] += c
            yield os.path.basename(path), parts[0], parts[2] if len(parts) > 2 else ""


def test_m0_is_the_compilers():
    """Loads to LDS get m0 as an operand, and no statement writes it: the compiler does not
    honour it among the clobbered registers."""
    found = list(statements())
    loads = [s for s in found if "load_lds" in s[1]]
    assert len(found) > 5 and loads
    for name, code, inputs in loads:
        assert '"{m0}"' in inputs, (name, code)
    assert not [s for s in found if re.search(r"\bs_\w+\s+m0\s*,", s[1])]
