"""Index arithmetic of the decoding kernels that no ordinary size shows, read from the sources."""
import os
import re

from paper_2606_26650_gb300 import build


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return f.read()


def test_a_heads_offset_in_the_rotation_has_64_bits():
    """catq_rope_at accepts 65536 heads of 65536 elements: the last of them begins behind 2^31 elements."""
    body = re.search(r"void rotate_heads\(.*?\n}\n", source("kv_cache.cu"), re.S).group(0)
    offsets = re.findall(r"[xy] \+ ([^;]*?) \* d \+ q\.[ab]", body)
    assert len(offsets) == 4 and all(o == "static_cast<int64_t>(h + k)" for o in offsets)


def test_kernels_launched_beside_the_launch_ahead_load_coherently():
    """Kernels of the decode step are launched while the one ahead still runs; what they load may be what that one writes
    (page scales, activations), which a non-coherent load is not defined for."""
    for name in ("kv_cache.cu", "kv_attn_tc.cu", "rope.cuh", "ternary_infer.cu"):
        code = re.sub(r"//[^\n]*", "", source(name))
        for load in ("__ldg(", "ldg_hint(", "ld.global.nc"):
            assert load not in code, f"{name}: {load}"
