"""What the device code says to the compiler about its assembly, read from the sources (no GPU needed)."""
import glob
import os
import re

from paper_2602_06694_amd import build


def assembly():
    """(file, line, statement) of every asm statement in the sources."""
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.h")) + glob.glob(os.path.join(build.CSRC, "*.hip"))):
        text = open(path).read().replace("\\\n", "  ")
        for m in re.finditer(r"\basm\s+volatile\s*\(|\b__asm__\s+volatile\s*\(|\basm\s*\(", text):
            depth, at, quoted = 1, m.end(), False
            while depth:
                c = text[at]
                if c == '"' and text[at - 1] != "\\":
                    quoted = not quoted
                elif not quoted:
                    depth += (c == "(") - (c == ")")
                at += 1
            yield os.path.basename(path), text.count("\n", 0, m.start()) + 1, text[m.start():at]


def test_assembly_that_writes_m0_says_so():
    """The compiler keeps values of its own in m0 (indexed registers, messages): a statement that writes it has to name it among what it changes."""
    writers = [(f, line, s) for f, line, s in assembly() if re.search(r"\bs_\w+\s+m0\s*,", s)]
    assert len(writers) >= 2, "no statement found"
    silent = [(f, line) for f, line, s in writers if not re.search(r'"m0"\s*[,)]', s.split(":")[-1])]
    assert not silent, silent
