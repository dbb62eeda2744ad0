"""Wait states inside the kernels' assembly text, which the compiler does not look into (no GPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_10537_amd", "csrc")


def statements():
    """(file, line, instructions) of every asm statement that holds instructions."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*"))):
        text = open(path).read()
        for m in re.finditer(r'\basm(?:\s+volatile)?\s*\(\s*((?:"(?:[^"\\]|\\.)*"\s*|[A-Z_]+\s*)+)', text):
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1)))
            ops = [i.strip() for i in re.split(r"\\n|\\t|;", code) if i.strip()]
            if ops:
                yield os.path.basename(path), text.count("\n", 0, m.start()) + 1, ops


def test_direct_loads_wait_for_m0():
    """A direct load to LDS reads M0, which a scalar instruction right in front of it has not written yet: one instruction has to stand between, in the
    same statement (what the compiler puts in front of a statement is its own matter, so the write has to be in it too)."""
    seen, bad = 0, []
    for name, line, ops in statements():
        for k, op in enumerate(ops):
            if not re.match(r"(global_load_lds|buffer_load\S* .*\blds\b)", op):
                continue
            seen += 1
            writes = [j for j in range(k) if re.match(r"s_\w+\s+m0\b", ops[j])]
            if not writes or k - writes[-1] < 2:
                bad.append(f"{name}:{line}: {' ; '.join(ops)}")
    assert seen > 10 and not bad, "\n".join(bad)
