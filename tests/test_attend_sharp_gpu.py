"""Attention as sharp as its calls allow (GPU).

Rows and requests of whole numbers have whole distances, and fp32, bf16 and
4-bit rows, their products and norms hold these exactly. At beta >= 1000 the next
distance has a weight of e^-1000, which is 0 in 32 and in 64 bits: predictions
are means over the nearest rows, and lse is -beta * distance + log of their
number, whatever beta is.
"""
import math

import numpy as np
import pytest
import torch

import attend_ref as ref
from test_attend_gpu import DEV, forward

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
D = 128
BATCHES = [(9, 400), (70, 3000), (300, 20_011)]   # the last: bf16 by 256 x 256 tiles
BETAS = [1e3, 1e6, 3e9, 1e12, 1e20, 1e30]


def whole(dtype, B, N, M=3, seed=0, same=0):
    """Rows and requests of -1, 0 and 1; the first `same` requests are rows of the
    bank, rows 10 and 20 are the same."""
    import paper_2606_17949_amd as rb
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.randint(-1, 2, (N, D), generator=g, device=DEV).to(t)
    x[20] = x[10]
    q = torch.randint(-1, 2, (B, D), generator=g, device=DEV).to(t)
    if same:
        at = torch.randint(0, N, (same,), generator=g, device=DEV)
        at[0] = 10
        q[:same] = x[at]
    s = {"queries": q, "scales": None, "mask": None, "x": x.double(), "bank": x,
         "qual": torch.rand(N, M, generator=g, device=DEV),
         "len": torch.exp(5.0 + 0.6 * torch.randn(N, M, generator=g, device=DEV)),
         "dq_hat": torch.randn(B, M, generator=g, device=DEV),
         "dl_hat": torch.randn(B, M, generator=g, device=DEV) * 1e-2,
         "dlse": torch.randn(B, generator=g, device=DEV)}
    if dtype == "q4":
        s["bank"], s["scales"], s["norms"] = rb.rb_bank_pack(x)
        assert torch.equal(ref.unpack4(s["bank"], s["scales"]), s["x"])
    else:
        s["norms"] = rb.rb_bank_norms(x)
    qd = q.double()
    s["dist"] = (qd * qd).sum(1)[:, None] + (s["x"] * s["x"]).sum(1)[None] - 2.0 * qd @ s["x"].t()
    s["least"] = s["dist"].amin(1, keepdim=True)
    s["near"] = (s["dist"] == s["least"]).double()
    return s


@pytest.mark.parametrize("beta", BETAS)
@pytest.mark.parametrize("B,N", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_all_weight_on_the_nearest(dtype, B, N, beta):
    s = whole(dtype, B, N, seed=N)
    out = forward(s, beta)
    torch.cuda.synchronize()
    b = float(np.float32(beta))
    ties = s["near"].sum(1, keepdim=True)
    for k, v in (("q_hat", s["qual"].double()), ("l_hat", s["len"].double())):
        mean = s["near"] @ v / ties
        # weights of exactly 1; a sum of as many labels, one of weights, a division
        # and the joins' products (16 roundings of them)
        ref.check(k, out[k], mean, (ties + 16.0) * U * mean, f"{dtype} {beta}")
    lse = -b * s["least"][:, 0] + torch.log(ties[:, 0])
    # rounded once; the logarithm of the ties to a few roundings of itself
    ref.check("lse", out["lse"], lse, U * lse.abs() + 4.0 * U * (1.0 + torch.log(ties[:, 0])),
              f"{dtype} {beta}")
