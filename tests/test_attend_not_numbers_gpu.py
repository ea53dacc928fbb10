"""Labels, rows and requests that are no numbers and are not masked (GPU): they
show in the predictions that they enter, and in no others, alike for every type
and size of batch."""
import math

import pytest
import torch

import attend_ref as ref
from test_attend_gpu import DEV, forward, make

pytestmark = pytest.mark.gpu

# batches of one tile, of several, and (bf16) of products of 256 x 256 tiles
BATCHES = [(3, 500), (70, 3000), (300, 20_011)]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("M", [3, 8, 9])
@pytest.mark.parametrize("B,N", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_labels_that_are_no_numbers(dtype, B, N, M, masked):
    """At beta = 3 every weight is well above 0 (e^-12 of the largest at least), so
    that a column with an infinite label is infinite and one with NaN, or with
    infinities of both signs, is NaN. All other columns keep their bits."""
    s = make(dtype, B, N, 128, M, mask="some" if masked else None)
    live = torch.nonzero(torch.ones(N, device=DEV) if s["mask"] is None else s["mask"])[:, 0]
    at = [int(live[i]) for i in (0, len(live) // 3, len(live) // 2, len(live) - 1)]
    for k in ("qual", "len"):
        s[k][at] = 1.0
    want = forward(s, 3.0)
    s["qual"][at[1], 0] = math.nan
    s["qual"][at[0], 1] = math.inf
    s["qual"][at[3], 2] = -math.inf
    s["len"][at[2], 0] = math.inf
    s["len"][at[3], 0] = -math.inf
    s["len"][at[2], M - 1] = math.inf
    got = forward(s, 3.0)
    torch.cuda.synchronize()
    for k, m, v in (("q_hat", 0, math.nan), ("q_hat", 1, math.inf), ("q_hat", 2, -math.inf),
                    ("l_hat", 0, math.nan), ("l_hat", M - 1, math.inf)):
        want[k][:, m] = v
    for k in want:
        assert torch.equal(torch.nan_to_num(got[k], 7.5, 1e38, -1e38),
                           torch.nan_to_num(want[k], 7.5, 1e38, -1e38)), k


@pytest.mark.parametrize("which", ["all", "first tile", "half a tile", "one"])
@pytest.mark.parametrize("B,N", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_rows_that_are_no_numbers(dtype, B, N, which):
    """One distance that is no number makes the softmax none, also where a wave or
    a tile has no other rows."""
    s = make(dtype, B, N, 128, 3)
    rows = {"all": slice(0, N), "first tile": slice(0, 256), "half a tile": slice(128, 256),
            "one": slice(N - 1, N)}[which]
    s["norms"][rows] = math.nan
    if dtype != "q4":
        s["bank"][rows] = math.nan
    out = forward(s, 4.0)
    torch.cuda.synchronize()
    for k, v in out.items():
        assert torch.isnan(v).all(), k


@pytest.mark.parametrize("B,N", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_a_request_that_is_no_number(dtype, B, N):
    s = make(dtype, B, N, 128, 3, mask="some")
    s["queries"][B // 2, 5] = math.nan
    out = forward(s, 4.0)
    torch.cuda.synchronize()
    for k, (value, bound) in ref.attend(s["queries"], s["x"], 4.0, s["qual"], s["len"],
                                        s["mask"]).items():
        assert torch.isnan(value[B // 2]).all() and torch.isnan(out[k][B // 2]).all(), k
        others = torch.arange(B, device=DEV) != B // 2
        ref.check(k, out[k][others], value[others], bound[others], dtype)
