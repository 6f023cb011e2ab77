"""What the losses' sources are held to, for the routed layer's and the clipping's: waits around the loads that are written in assembly, and accesses as
another type than was written."""
import os
import re
import subprocess

from paper_1901_01544_amd import build
from test_lds_load_waits import code, too_close

CSRC = os.path.join(build.HERE, "csrc")


def test_waits_around_the_loads(tmp_path):
    source = next(s for s in build.SOURCES if s.endswith("iwp_experts.hip"))
    out = str(tmp_path / "experts.s")
    done = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-S", "-o", out, source], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-2000:]
    loads = 0
    for function in re.split(r"\n(?=_ZN3iwp\w+:)", open(out).read())[1:]:
        lines = code(function.split(".Lfunc_end")[0])
        n, found = too_close(lines)
        assert not found, found[:3]
        loads += n
        assert all(l.startswith("s_mov_b32 m0,") for l in lines if re.search(r"\bm0\b", l))
    assert loads > 100


def test_casts_of_pointers():
    """Only to types that may alias any other, to char, or to an element's own type where a caller's row is at hand as char or what a kernel's
    own LDS or workspace holds is of that type throughout, or from one fence to the next (the routing's LDS)."""
    shared = open(os.path.join(CSRC, "iwp_matrix.hpp")).read()
    text = "".join(open(os.path.join(CSRC, n)).read() for n in ("iwp_tokens.hpp", "iwp_route.hpp", "iwp_grouped.hpp", "iwp_experts.hip", "iwp_clip.hip"))
    alias = set(re.findall(r"typedef \w+ (\w+) __attribute__\(\([^;]*\bmay_alias\b[^;]*\)\);", shared + text))
    casts = set(re.findall(r"reinterpret_cast<(?:const )?(\w+)\s*\*>", text)) - alias
    assert casts == {"char", "uint16_t", "uint32_t", "f32x4", "T", "Candidate", "SlotGradient", "float", "double", "int32_t"}
