"""The losses' kernels write bytes as one type and read them as another: every such access goes through a type that may alias any other, since the
build does not switch the type-based analysis off."""
import os
import re

from paper_1901_01544_amd import build

CSRC = os.path.join(build.HERE, "csrc")


def test_casts_of_pointers():
    text = "".join(open(os.path.join(CSRC, n)).read() for n in ("iwp_matrix.hpp", "iwp_head.hpp", "iwp_balance.hpp", "iwp_losses.hip"))
    alias = set(re.findall(r"typedef \w+ (\w+) __attribute__\(\([^;]*\bmay_alias\b[^;]*\)\);", text))
    assert alias
    casts = re.findall(r"reinterpret_cast<(?:const )?(\w+)\s*\*>", text)
    assert len(casts) > 20
    # char may alias anything; s16x8 and f32x4 are read where the same type, or no instruction that the compiler knows of, wrote; elements of
    # 16 and 32 bits are single ones of a caller's row, whose bytes are at hand as char
    assert set(casts) - alias == {"char", "s16x8", "f32x4", "uint16_t", "uint32_t", "T"}
    for target in ("uint16_t", "uint32_t"):
        for at in re.findall(r"reinterpret_cast<(?:const )?%s\*>\((\w+)\)" % target, text):
            assert re.search(r"char\* %s = static_cast<(?:const )?char\*>" % at, text), at
