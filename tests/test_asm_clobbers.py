"""What the assembly statements of the sources overwrite, they name."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_08756_amd", "csrc")


def _statements():
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", text, flags=re.S):
            yield name, m[1]


def test_statements_that_write_m0_name_it_as_overwritten():
    writers = [(n, s) for n, s in _statements() if re.search(r"\bs_mov_b32 m0\b", s)]
    assert writers
    for name, s in writers:
        assert '"m0"' in s.rsplit(":", 1)[1], (name, s)
