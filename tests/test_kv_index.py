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


def test_three_terms_of_a_weight():
    """The attention's weights as three e5m2 terms, restated: every fp16 number up to 2^15.75 within 2^-9 of itself (with its own
    rounding from fp32, 2^-11), or half of the last term's least step, and none of the terms behind the first leans to a side."""
    import numpy as np
    code = source("kv_attn_tc.cu")
    units = [float(x) for x in re.search(r"kUnitM = ([0-9.]+)f, kUnitL = ([0-9.]+)f", code).groups()]
    x = np.arange(0x7C00, dtype=np.uint16).view(np.float16)
    exact = x.astype(float)
    x, exact = x[exact <= 2.0 ** 15.75], exact[exact <= 2.0 ** 15.75]

    def cut(v):
        return (v.view(np.uint16) & 0xFF00).view(np.float16)

    def rounded(v):
        return cut((v.view(np.uint16) + np.uint16(0x80)).view(np.float16))

    for (um, ul), floor in ((units, 2.0 ** -23), ((1.0, 1.0), 2.0 ** -17)):
        h = rounded(x)
        b = (x - h) * np.float16(1 / um)
        c = (b - cut(b)) * np.float16(um / ul)
        terms = [t.astype(float) * u for t, u in zip((h, cut(b), rounded(c)), (1.0, um, ul))]
        assert all(np.isfinite(t).all() for t in terms)
        assert (np.abs(sum(terms) - exact) <= np.maximum((2.0 ** -9 - 2.0 ** -11) * exact, floor)).all()
        big = exact > 2.0 ** -6
        for t in terms[1:]:
            assert abs((t[big] / exact[big]).mean()) <= 2.0 ** -9
