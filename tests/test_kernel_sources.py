"""Device functions of the kernels' headers: one body for a name and its arguments, whichever files include them."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_21428_b200", "csrc")
FUNCTION = re.compile(r"__device__ (?:__forceinline__|inline) [\w:<>, *]+?[ *&](\w+)\(([^{;]*?)\)\s*\{")


def test_headers_define_a_device_function_once():
    seen = {}
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cuh", ".h")):
            continue
        for function, arguments in FUNCTION.findall(open(os.path.join(CSRC, name)).read()):
            types = tuple(re.sub(r"\s*\(?[&*]?\w+\)?(\[\d+\])?$", "", a.strip()) for a in arguments.split(","))
            seen.setdefault((function, types), set()).add(name)
    assert len(seen) > 60
    assert not {k: v for k, v in seen.items() if len(v) > 1}
