"""Attention of whole prompts where the arithmetic is at its ends, against its definition in 64 bits."""
import math

import pytest
import torch

from kv4_reference import HALF
from paper_2207_08820_b200 import api
from test_gpu_prompt import BF16, F16, ints, reference

pytestmark = pytest.mark.gpu


def reference_of_all_weights(q, k, v, scale):
    """As reference(), every row over all keys, where weights below fp16's normal numbers keep their bits down to 2^-32 of the row's largest."""
    u, D, m = HALF[q.dtype], q.shape[-1], k.shape[0]
    out, far = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for h in range(q.shape[1]):
        qd, kd, vd = q[:, h].double(), k[:, h].double(), v[:, h].double()
        a = scale * (qd @ kd.T)
        p = torch.softmax(a, 1)
        out[:, h] = p @ vd
        # scores: D / 16 additions in the tensor core, three roundings, of them and of the maximum they are compared with; the exponential 2^-20; the weight's own rounding; sums
        size = scale * (qd.abs() @ kd.abs().T)
        off = size * (D / 16 + 4) * 2.0 ** -23 + 4 * 2.0 ** -24 * size.amax(1, keepdim=True)
        rel = torch.expm1((off + off.amax(1, keepdim=True)).clamp(max=50)) + 2.0 ** -20
        bound = (p * (rel + (p * rel).sum(1, keepdim=True) + u + (m / 16 + 8) * 2.0 ** -23)) @ vd.abs()
        bound = bound + 2.0 ** -32 * p.amax(1, keepdim=True) * vd.abs().sum(0)
        far[:, h] = bound + u * (out[:, h].abs() + bound) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
    return out, far


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("power", [-8, -14, -18, -22])
@pytest.mark.parametrize("where", [0, 300, 599])
def test_large_values_of_little_weight(where, power, dtype):
    """One key has nearly all of the weight and a small value; the others' values make up for their weights."""
    n, D = 600, 64
    gen = torch.Generator("cuda").manual_seed(1)
    q = torch.zeros(130, 2, D, dtype=dtype, device="cuda")
    q[..., 0] = 1
    k = (torch.randn(n, 2, D, device="cuda", generator=gen) * 0.5).to(dtype)
    k[where, :, 0] = -power * math.log(2) + 2          # 2^power and less for the others
    v = (torch.randn(n, 2, D, device="cuda", generator=gen) * min(2.0 ** -power, 2.0 ** 13)).to(dtype)
    v[where] = 2.0 ** -10
    out = api.attend_prompt(q, k, v, ints([0, 130]), ints([0, n]), causal=False, scale=1.0)
    want, far = reference_of_all_weights(q, k, v, 1.0)
    off = (out.double() - want).abs()
    assert (off <= far).all(), (off.max(), (off / far).max())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scale", [1e-44, 1e-38, 1e-20, 1e20, 2.3e38])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_scales_near_the_ends_of_binary32(dtype, scale, causal):
    """Queries of zeros see the mean of the values whatever the scale is, and so do all where the scale leaves nothing of the scores."""
    gen = torch.Generator("cuda").manual_seed(2)
    k, v = (torch.randn(300, 2, 96, device="cuda", generator=gen).to(dtype) for _ in range(2))
    q = torch.zeros(300, 4, 96, dtype=dtype, device="cuda")
    if scale < 1:
        q[::2] = torch.randn(150, 4, 96, device="cuda", generator=gen).to(dtype)
    want, far = reference(q, k, v, causal, scale)
    assert ((api.attend_prompt(q, k, v, causal=causal, scale=scale).double() - want).abs() <= far).all()


@pytest.mark.parametrize("power", [-110, -60, 60, 100])
def test_scales_that_make_up_for_the_size_of_queries(power):
    gen = torch.Generator("cuda").manual_seed(3)
    q, k, v = ((torch.randn(300, 2, 128, device="cuda", generator=gen) * s).to(BF16) for s in (2.0 ** power, 1.0, 1.0))
    scale = 2.0 ** -power / 128 ** 0.5
    want, far = reference(q, k, v, True, scale)
    assert ((api.attend_prompt(q, k, v, scale=scale).double() - want).abs() <= far).all()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("power,gap", [(0, 1), (16, 1), (20, 1), (22, 1), (24, 2), (26, 8), (28, 32), (30, 128)])
def test_large_scores(power, gap, order, dtype):
    """Scores that binary32 holds exactly, 2^power and a few gaps more or less: what sets them apart counts, whatever their size."""
    n, D = 600, 64
    gen = torch.Generator("cuda").manual_seed(4)
    steps = torch.arange(n, device="cuda") // 40 if order != "mixed" else torch.randint(0, 15, (n,), device="cuda", generator=gen)
    steps = 15 - steps if order == "down" else steps
    q, k = torch.zeros(70, 1, D, dtype=dtype, device="cuda"), torch.zeros(n, 1, D, dtype=dtype, device="cuda")
    q[..., 0], k[..., 0], q[..., 1], k[:, 0, 1] = 2.0 ** (power // 2), 2.0 ** (power - power // 2), float(gap), steps.to(dtype)
    q[35:, :, 0] *= -1          # and far below zero
    v = torch.randn(n, 1, D, device="cuda", generator=gen).to(dtype)
    out = api.attend_prompt(q, k, v, ints([0, 70]), ints([0, n]), causal=False, scale=1.0).double()[:, 0]
    p = torch.softmax(gap * steps.double(), 0)
    want = (p @ v[:, 0].double()).expand(70, D)
    # distances of up to 15 gaps times log2(e), rounded: 2^-17 of a weight and less, for those that leave one.  Below 2^20 scores may be rounded before their distance is
    # taken, by 2^(power - 23), for all of a row alike until its maximum is replaced: then for weights that are 2^-8 of the largest and less.  The exponential 2^-20
    u = HALF[dtype]
    rel = 2.0 ** -17 + (2.0 ** (power - 22 - 8) if power < 20 else 0.0)
    bound = (2 * rel + u + (n / 16 + 8) * 2.0 ** -23) * (p @ v[:, 0].double().abs()) + 2.0 ** -32 * p.max() * v[:, 0].double().abs().sum(0)
    far = bound + u * (want.abs() + bound)
    off = (out - want).abs()
    assert (off <= far).all(), (off.max(), (off / far).max())
