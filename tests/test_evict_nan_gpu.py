"""Eviction by usage that is no number (GPU): last, whatever the sign and the
payload, and in the order of the rows."""
import numpy as np
import pytest
import torch

from test_bank_rows_gpu import victims_of

pytestmark = pytest.mark.gpu

DEV = "cuda"
# quiet and signalling, of both signs, least and greatest payloads
NANS = np.array([0x7fc00000, 0xffc00000, 0x7f800001, 0xff800001, 0x7fffffff, 0xffffffff],
                np.uint32)


def evict(u, n, may=None):
    import paper_2606_17949_amd as rb
    got = rb.rb_bank_evict(torch.from_numpy(u).to(DEV), n,
                           may_go=None if may is None else torch.from_numpy(may).to(DEV))
    torch.cuda.synchronize()
    return got.cpu().numpy()


@pytest.mark.parametrize("bits", [int(b) for b in NANS])
def test_a_nan_goes_last(bits):
    u = np.array([0.0, 3.0, np.inf, -np.inf, 1.0, -0.0, 0.0, -2.0], np.float32)
    u.view(np.uint32)[0] = bits
    for n in range(1, 9):
        assert np.array_equal(evict(u, n), victims_of(u, None, n)), n


@pytest.mark.parametrize("share", [0.05, 0.9, 1.0])
@pytest.mark.parametrize("N", [7, 5000, 20_000, 300_001])
def test_many_nans(N, share):
    r = np.random.RandomState(N)
    u = r.standard_normal(N).astype(np.float32)
    u[r.rand(N) < 0.02] = np.inf
    u[r.rand(N) < 0.02] = -np.inf
    nan = r.rand(N) < share
    u.view(np.uint32)[nan] = r.choice(NANS, int(nan.sum()))
    numbers = int((~np.isnan(u)).sum())
    for n in sorted({1, max(1, numbers // 2), numbers, min(N, numbers + 1), (numbers + N) // 2, N}):
        if n > 0:
            assert np.array_equal(evict(u, n), victims_of(u, None, n)), n
    may = (r.rand(N) < 0.5).astype(np.uint8)
    n = max(1, N // 3)
    assert np.array_equal(evict(u, n, may), victims_of(u, may, n))
