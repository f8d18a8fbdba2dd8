"""The rules on logits in their own place: bit for bit what a call with another output gives, at sizes on both sides of the small stretches, and nothing
outside the rows."""
import numpy as np
import pytest
import torch

import detsynth as ds
from gpu_util import DEV, step, up
from test_gpu_logits import d, rules_of, run  # noqa: F401 (fixture among them)

pytestmark = pytest.mark.gpu

# vectors of 16 bytes times rows: from 2^18 on a stretch is 4096 tokens (66 x 32003 of fp32, 140 x 32003 and 33 x 64003 of bf16), else 1024 or 2048
FP32 = [(1, 1, 1), (2, 33, 9), (5, 1025, 300), (7, 32001, 700), (64, 8190, 33), (66, 32003, 300), (9, 128000, 4001), (33, 32768, 50)]
BF16 = [(1, 1, 1), (2, 33, 9), (5, 2049, 300), (7, 32001, 700), (66, 32003, 300), (140, 32003, 90), (33, 64003, 1000), (64, 32768, 50)]


def place(z, pad, fill):
    """z's rows `pad` elements apart in a wider tensor of `fill`; its first rows hold z."""
    B, V = z.shape
    wide = torch.full((B, V + pad), fill, dtype=z.dtype, device=DEV)
    wide[:, :V] = z
    return wide


def bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("parts", ["all", "penalties", "biases", "masks", "none"])
@pytest.mark.parametrize("dtype,B,V,T", [(torch.float32, *s) for s in FP32] + [(torch.bfloat16, *s) for s in BF16],
                         ids=[f"fp32-{B}x{V}" for B, V, _ in FP32] + [f"bf16-{B}x{V}" for B, V, _ in BF16])
def test_in_place_as_apart(d, dtype, B, V, T, parts):  # noqa: F811
    rng = np.random.default_rng(B * 1000 + V + 7)
    on = lambda w: parts in ("all", w)  # noqa: E731
    h = rules_of(rng, B, V, T, on("penalties"), 6 * on("biases"), 3 * on("masks"))
    host = rng.normal(0, 3, (B, V)).astype(np.float32)
    host.ravel()[::7], host.ravel()[3::11], host.ravel()[5::97], host.ravel()[6::89] = 0.0, -0.0, np.inf, -np.inf
    z = up(host) if dtype == torch.float32 else ds.to_torch_bf16(ds.f32_to_bf16_bits(host), DEV)
    bits(z).view(-1)[::13] = 0x7FA1 << (16 if dtype == torch.float32 else 0)      # a NaN with a payload
    step(f"{dtype} {B} rows of {V}, {parts}")
    want = run(d, z, h)
    if parts == "none":
        assert torch.equal(bits(want), bits(z))
    for pad in (0, 5, 64):
        wide = place(z, pad, 5.0)
        run(d, wide[:, :V], h, wide[:, :V])
        assert torch.equal(bits(wide[:, :V]), bits(want)) and (wide[:, V:] == 5).all()
