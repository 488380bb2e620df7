"""Appending promises the bits of rope and store one behind the other.  Both kernels turn pairs with the same functions, whose
roundings are written down: checked on the sources, since equal results show only what one compiler made of them."""
import os
import re

import pytest

from paper_2502_03805_b200 import build


def source(name):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(build.CSRC, name)).read(), flags=re.S)


@pytest.mark.parametrize("name", ["rope.cu", "append.cu"])
def test_cosines_and_sines_enter_nothing_but_the_shared_sums(name):
    text = source(name)
    assert '#include "rotate.cuh"' in text and not re.search(r"float\s+turned_(first|second)", text)
    rest = re.sub(r"turned_(first|second)\((?:[^()]|\([^()]*\))*\)", "", text)     # the sums' arguments
    assert len(re.findall(r"turned_first\(", text)) == len(re.findall(r"turned_second\(", text)) >= 1
    uses = re.findall(r"[^;{}\n]*\b(?:cs|sn)\[[^;{}\n]*", rest)
    for use in uses:
        assert re.fullmatch(r"\s*(float cs\[P\], sn\[P\]|sincospif\(.*&sn\[i\], &cs\[i\]\)|(cs|sn)\[i\] \*= p\.factor)\s*", use), use
    assert uses


def test_the_shared_sums_round_explicitly():
    body = source("rotate.cuh")
    code = body[body.index("{", body.index("float turned_first")):]
    assert "__fmaf_rn" in code and "__fmul_rn" in code
    assert not re.search(r"\w\s*[*+]\s*\w", re.sub(r"float (turned_\w+)\([^)]*\)", "", code))
