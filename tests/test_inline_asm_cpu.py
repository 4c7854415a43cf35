"""Inline assembly in the kernels names what it writes (CPU only)."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_21137_amd", "csrc")


def _statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"\basm\s+volatile\s*\(", text):
            depth, i, quoted = 1, m.end(), False
            while depth:
                c = text[i]
                quoted ^= c == '"' and text[i - 1] != "\\"
                depth += 0 if quoted else (c == "(") - (c == ")")
                i += 1
            body = text[m.end():i - 1]
            parts, at = [""], 0
            for piece in re.findall(r'"(?:\\.|[^"\\])*"|::|:|[^":]+', body):
                if piece in (":", "::"):
                    parts += [""] * len(piece)
                else:
                    parts[-1] += piece
            yield os.path.basename(path), parts[0].replace("\\n", "\n").replace("\\t", "\t"), parts[3] if len(parts) > 3 else ""


def test_what_is_written_is_named():
    seen = 0
    for name, code, clobbers in _statements():
        if re.search(r"\bm0\s*,", code):
            assert '"m0"' in clobbers, f"{name}: {code}"
            seen += 1
        if re.search(r"\bbuffer_load\w*[^\n]*\blds\b|\bds_write|\b(global|buffer|flat)_(store|atomic)", code):
            assert '"memory"' in clobbers, f"{name}: {code}"
            seen += 1
    assert seen >= 2
