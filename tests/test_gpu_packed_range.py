"""The packed attention with values of far magnitudes: weighted sums are fp32 and
divided by their weights' sum at the end, so values below 2^80 give finite results,
also where the scores rise from tile to tile and the running maximum with them."""
import numpy as np
import pytest

from oracle import heads as O
from helpers import dev, host
from test_gpu_heads import E, U, close, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [0.002, 0.05, 2.0])
def test_values_below_2_to_80(gpu, dtype, d, rise):
    import torch
    rng = np.random.default_rng(1)
    n = 700
    q = np.ones((n, 2, d), np.float32)
    k = host(dev(np.broadcast_to(np.arange(n)[:, None, None] * rise / d, (n, 1, d)), dtype))
    v = draw(rng, (n, 1, d), dtype)
    v = host(dev(v / np.abs(v).max() * 2.0 ** 80 * (1 - 2.0 ** -7), dtype))
    cfg = gpu.heads_config(2, 1, d, dtype=dtype, norm=False, rot_dim=0)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    x = [dev(y, dtype) for y in (q, k, v)]
    out, lse = gpu.packed_attention_forward(cfg, *x, cu, n, scale=1.0)
    ref, rl, err, mag = O.packed_attention(q, k, v, [0, n], 1.0)
    s = (d + 10) * E * err + 8 * E
    w = 2.0 ** -8 if dtype == "bf16" else 0.0
    close(host(out), ref, U[dtype] * np.abs(ref) + (2 * s + (n + 64) * E + w)[..., None] * mag, rise)
    close(host(lse), rl, 2 * s + (n + 64) * E + 4 * E * np.abs(rl), rise)
    do = dev(draw(rng, (n, 2, d), dtype), dtype)
    for y in gpu.packed_attention_backward(cfg, *x, out, lse, do, cu, n, scale=1.0):
        assert torch.isfinite(y).all()
