"""Large bf16 batches, which go by as products of 256 x 256 tiles (GPU): long rows,
label columns of several tiles, and masks that leave tiles and halves of tiles
without a row."""
import math

import pytest
import torch

import attend_ref as ref
from test_attend_gpu import DEV, backward, dirty, forward, make

pytestmark = pytest.mark.gpu


def takes_tiles(B, N, d, M):
    """The rule of at_gemm (tests/test_attend_plan.py) on this device."""
    cu = torch.cuda.get_device_properties(0).multi_processor_count
    return (d >= 128 and B > 128 and 2 * -(-N // 256) * -(-B // 256) >= cu and
            (-(-2 * M // 16) < 2 * -(-2 * M // 32) or d > 1280))


def check_all(got, want, label):
    for k, (value, bound) in want.items():
        half = torch.finfo(got[k].dtype).eps / 2 if got[k].dtype == torch.bfloat16 else 0.0
        print(k, ref.check(k, got[k], value, bound + half * value.abs() + ref.T, label), flush=True)


def usage(s, beta, lse, old, **kw):
    import paper_2606_17949_amd as rb
    use = old.clone()
    rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], beta, lse, use, decay=0.75,
                       row_mask=s["mask"], **kw)
    return use


def check_usage(s, beta, lse, label):
    old = torch.rand(s["norms"].shape[0], device=DEV)
    value, bound = ref.usage(s["queries"], s["x"], beta, lse, old, 0.75, s["mask"])
    print("usage", ref.check("usage", usage(s, beta, lse, old), value, bound, label), flush=True)


@pytest.mark.parametrize("mask", [None, "some"])
@pytest.mark.parametrize("B,N,d,M,beta", [
    # rows of 3 to 32 stages, some ending inside one; one to five tiles of requests; 6 to
    # 34 label columns, the sum of the weights among them or not
    (130, 33_025, 264, 3, 12.0), (200, 33_000, 768, 4, 8.0), (300, 17_000, 2048, 9, 5.0),
    (129, 40_011, 1000, 17, 10.0), (300, 20_011, 200, 8, 5.0), (1025, 7000, 512, 7, 20.0),
    (257, 16_385, 136, 33, 3.0)])
def test_forward_and_usage(B, N, d, M, beta, mask):
    import paper_2606_17949_amd as rb
    assert takes_tiles(B, N, d, M)
    label = f"B={B} N={N} d={d} M={M} mask={mask}"
    print(label, flush=True)
    s = make("bf16", B, N, d, M, seed=B, mask=mask)
    out = forward(s, beta, ws=dirty(rb.rb_attend_workspace_size(B, N, d, rb.RB_BF16, M)))
    check_all(out, ref.attend(s["queries"], s["x"], beta, s["qual"], s["len"], s["mask"]), label)
    check_usage(s, beta, out["lse"], label)


def masked(s, live):
    """The rows that are not live hold no numbers, and are masked."""
    dead = ~live
    s["mask"] = live.to(torch.uint8)
    s["bank"][dead], s["norms"][dead], s["len"][dead] = math.nan, math.nan, math.nan
    s["qual"][dead] = math.inf
    return s


@pytest.mark.parametrize("which", ["tiles and halves", "one row", "one row of the last tile",
                                   "first half of the first tile", "every 300th row"])
@pytest.mark.parametrize("M", [3, 8])
def test_tiles_without_rows(which, M):
    B, N, d = 300, 20_011, 128
    assert takes_tiles(B, N, d, M)
    s = make("bf16", B, N, d, M)
    live = torch.zeros(N, dtype=torch.bool, device=DEV)
    if which == "tiles and halves":
        live[:] = True
        live[:512] = live[640:768] = live[1024:1152] = live[N - 43:] = False
    elif which == "one row":
        live[700] = True
    elif which == "one row of the last tile":
        live[N - 1] = True
    elif which == "first half of the first tile":
        live[:128] = True
    else:
        live[::300] = True
    masked(s, live)
    out = forward(s, 5.0)
    check_all(out, ref.attend(s["queries"], s["x"], 5.0, s["qual"], s["len"], s["mask"]), which)
    check_usage(s, 5.0, out["lse"], which)
    got = backward(s, 5.0, out)
    check_all(got, ref.backward(s["queries"], s["x"], 5.0, s["qual"], s["len"], out["q_hat"],
                                out["l_hat"], out["lse"], s["dq_hat"], s["dl_hat"], s["dlse"],
                                s["mask"]), which)


@pytest.mark.parametrize("M", [3, 8])
def test_no_row_left(M):
    B, N = 300, 20_011
    assert takes_tiles(B, N, 128, M)
    s = masked(make("bf16", B, N, 128, M), torch.zeros(N, dtype=torch.bool, device=DEV))
    out = forward(s, 4.0)
    assert torch.isnan(out["q_hat"]).all() and torch.isnan(out["l_hat"]).all()
    assert torch.isneginf(out["lse"]).all()
    old = torch.rand(N, device=DEV)
    assert torch.equal(usage(s, 4.0, out["lse"], old), old * 0.75)
    for k, v in backward(s, 4.0, out).items():
        assert torch.count_nonzero(v) == 0, k


def test_some_requests_dead():
    """Requests without weights (lse -inf given) add nothing to the rows' usage."""
    B, N = 300, 20_011
    s = make("bf16", B, N, 128, 3, mask="some")
    out = forward(s, 4.0)
    out["lse"][[0, 7, 63, 64, 255, 256, 299]] = -math.inf
    check_usage(s, 4.0, out["lse"], "some dead")


def test_same_bits_every_time():
    B, N = 300, 20_011
    s = make("bf16", B, N, 200, 5, mask="some")
    first = forward(s, 5.0)
    old = torch.rand(N, device=DEV)
    use = usage(s, 5.0, first["lse"], old)
    for _ in range(3):
        again = forward(s, 5.0)
        for k in first:
            assert torch.equal(first[k], again[k]), k
        assert torch.equal(use, usage(s, 5.0, first["lse"], old))
