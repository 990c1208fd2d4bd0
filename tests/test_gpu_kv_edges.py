"""GPU tests of the decoding calls at the ends of their ranges, against the fp64 oracle: rows of more than 2^31 elements.

Tolerances, from the arithmetic: a rotation is off by 2^-22 (|a| + |b|) (sine and cosine within 2^-22.5, two products and a
sum in fp32) and half a step of the output's type."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from tests.test_gpu_kv import device, i32, rope_bound  # noqa: F401 (device: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_of_rows_past_32_bits(device, dtype):  # noqa: F811
    """One row of 40000 heads of 65536: a head's offset passes 2^31 elements from head 32768 on."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    nh, d, rot, pos = 40000, 65536, 64, 12345
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=device).manual_seed(5)
    X = torch.empty(1, nh * d, dtype=dt, device=device).normal_(generator=gen)
    rope = C.Rope.create(rot, 10000.0, device)
    Y = torch.zeros_like(X)
    C.catq_rope_at(X, i32([pos], device), rope, nh, d, Y)
    x, y = X.view(nh, d), Y.view(nh, d)
    assert torch.equal(x[:, rot:], y[:, rot:])  # what is not rotated passes unchanged
    freq, _ = K.frequencies(rot, 10000.0)
    host = x[:, :rot].float().cpu().numpy()[None].astype(np.float64)
    want = K.rope(host, np.array([pos]), freq, False)
    bound = rope_bound(host, freq, False, 1.0) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    got = y[:, :rot].float().cpu().numpy()[None]
    assert (np.abs(got - want) <= bound).all()
    C.catq_rope_at(X, i32([pos], device), rope, nh, d)  # in place
    assert torch.equal(X, Y)
    assert C.catq_device_status() == 0
    del X, Y, x, y
    torch.cuda.empty_cache()
