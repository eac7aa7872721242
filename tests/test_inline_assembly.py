"""Inline assembly names the registers that it changes, from the sources (no GPU needed)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_11418_amd", "csrc")


def _statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if path.endswith((".h", ".hip", ".cpp")):
            for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", open(path).read(), re.S):
                yield os.path.basename(path), m.group(1)


def test_m0_is_named_where_it_is_written():
    """The address that a load to LDS takes from m0 is set in the same statement: the compiler has to know that what it kept there is gone."""
    found = [(name, text) for name, text in _statements() if re.search(r"\bs_mov_b32\s+m0\b", text)]
    assert found
    for name, text in found:
        changed = text.rsplit(":", 1)[1]
        assert '"m0"' in changed and '"memory"' in changed, (name, text)
