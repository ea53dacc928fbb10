"""4-bit rows, eviction and replacement against plain numpy and torch (GPU)."""
import math

import numpy as np
import pytest
import torch

import attend_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"


def hold4(x):
    """Codes and scales by the rule, one element at a time in 64 bits (numpy)."""
    N, d = x.shape
    codes = np.zeros((N, d), np.uint8)
    scales = np.zeros((N, d // 32), np.uint8)
    mags = np.array(ref.MAGNITUDES)
    for n in range(N):
        for j in range(d // 32):
            g = x[n, 32 * j:32 * j + 32].astype(np.float64)
            top = np.abs(g).max()
            s = 1
            while s < 254 and top > 6.0 * 2.0 ** (s - 127):
                s += 1
            scales[n, j] = s
            y = g / 2.0 ** (s - 127)
            for i, v in enumerate(y):
                off = np.abs(mags - abs(v))
                near = np.flatnonzero(off == off.min())
                c = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
                codes[n, 32 * j + i] = c | (8 if np.signbit(g[i]) else 0)
    return codes[:, 0::2] | (codes[:, 1::2] << 4), scales


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,d", [(1, 32), (5, 96), (3, 512), (7, 544), (2, 2048)])
def test_pack(dtype, N, d):
    import paper_2606_17949_amd as rb
    g = torch.Generator().manual_seed(N * d)
    x = torch.randn(N, d, generator=g) * torch.exp2(
        torch.randint(-40, 40, (N, 1), generator=g).float())
    # ties between two elements, zeros of both signs, a group of nothing
    x[0, :16] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25,
                              -5.0, 0.0, -0.0, 0.26, 5.01])
    if d >= 64:
        x[N - 1, 32:64] = 0.0
    x = x.to(dtype)
    rows, scales, norms = rb.rb_bank_pack(x.to(DEV))
    torch.cuda.synchronize()
    codes, sc = hold4(x.float().numpy())
    assert np.array_equal(scales.cpu().numpy(), sc)
    assert np.array_equal(rows.cpu().numpy(), codes)
    v = ref.unpack4(rows, scales)
    want = (v * v).sum(1)
    # d squares (exact in 32 bits but for their sum): d roundings at most
    assert ((norms.double() - want).abs() <= d * 2.0 ** -24 * want).all()


def victims_of(usage, may_go, n):
    rows = np.arange(len(usage)) if may_go is None else np.flatnonzero(may_go)
    u = usage[rows].astype(np.float64) + 0.0
    u = np.where(np.isnan(u), np.inf, u)
    nan = np.isnan(usage[rows])
    order = np.lexsort((rows, nan, u))[:n]
    out = np.sort(rows[order])
    return np.concatenate((out, np.full(n - len(out), -1, out.dtype))).astype(np.int32)


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "falling", "wide"])
@pytest.mark.parametrize("N,n", [(1, 1), (2, 1), (63, 63), (1000, 0), (1000, 1), (8191, 100),
                                 (8193, 8193), (20_000, 5000), (300_001, 37), (300_001, 150_000)])
def test_evict(N, n, kind):
    import paper_2606_17949_amd as rb
    r = np.random.RandomState(N + n)
    u = {"random": lambda: r.exponential(size=N), "ties": lambda: r.randint(0, 7, N) * 0.5,
         "equal": lambda: np.full(N, 0.25), "falling": lambda: np.arange(N, 0, -1) * 1e-3,
         "wide": lambda: np.exp(r.uniform(-80, 80, N)) * r.choice([-1, 1], N)}[kind]()
    u = u.astype(np.float32)
    u[r.rand(N) < 0.05] = 0.0
    u[r.rand(N) < 0.05] = -0.0
    for may in (None, (r.rand(N) < 0.6).astype(np.uint8), np.zeros(N, np.uint8)):
        if may is not None and kind == "random":
            may = may * 3   # (any value but 0)
        ws = torch.full((rb.rb_evict_workspace_size(N),), 0xff, dtype=torch.uint8, device=DEV)
        got = rb.rb_bank_evict(torch.from_numpy(u).to(DEV), n,
                               may_go=None if may is None else torch.from_numpy(may).to(DEV),
                               ws=ws)
        torch.cuda.synchronize()
        assert np.array_equal(got.cpu().numpy(), victims_of(u, may, n))


def test_evict_no_numbers_last():
    import paper_2606_17949_amd as rb
    u = np.array([math.nan, 3.0, math.inf, -math.inf, 1.0, -0.0, 0.0], np.float32)
    for n in range(1, 8):
        got = rb.rb_bank_evict(torch.from_numpy(u).to(DEV), n)
        assert np.array_equal(got.cpu().numpy(), victims_of(u, None, n))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
@pytest.mark.parametrize("N,n,d,M", [(1, 1, 32, 1), (50, 7, 96, 3), (400, 400, 544, 20),
                                     (1000, 9, 2048, 4)])
def test_replace(dtype, N, n, d, M):
    import paper_2606_17949_amd as rb
    g = torch.Generator(device=DEV).manual_seed(N)
    src = torch.float32 if dtype == "f32" else torch.bfloat16
    bank = torch.randn(N, d, generator=g, device=DEV).to(src)
    scales = None
    if dtype == "q4":
        bank, scales, norms = rb.rb_bank_pack(bank)
    else:
        norms = rb.rb_bank_norms(bank)
    qual, ln = (torch.rand(N, M, generator=g, device=DEV) for _ in range(2))
    usage = torch.rand(N, generator=g, device=DEV)
    new = torch.randn(n, d, generator=g, device=DEV).to(src)
    nq, nl = (torch.rand(n, M, generator=g, device=DEV) for _ in range(2))
    at = torch.randperm(N, generator=g, device=DEV)[:n].to(torch.int32)
    if n > 2:
        at[1], at[2] = -1, N       # passed over
    state = [bank, norms, qual, ln, usage] + ([scales] if scales is not None else [])
    want = [t.clone() for t in state]
    inside = (at >= 0) & (at < N)
    rows = at[inside].long()
    if dtype == "q4":
        pr, ps, pn = rb.rb_bank_pack(new)
    else:
        pr, ps, pn = new, None, rb.rb_bank_norms(new)
    for t, v in zip(want, [pr, pn, nq, nl, torch.full((n,), 0.5, device=DEV)] +
                    ([ps] if ps is not None else [])):
        t[rows] = v[inside]
    rb.rb_bank_replace(at, new, nq, nl, bank, norms, qual, ln, scales=scales, usage=usage,
                       usage0=0.5)
    torch.cuda.synchronize()
    for t, w in zip(state, want):
        assert torch.equal(t, w)


def test_replace_fp32_rows_of_a_4_bit_bank():
    import paper_2606_17949_amd as rb
    x = torch.randn(40, 64, device=DEV)
    rows, scales, norms = rb.rb_bank_pack(x)
    z = torch.zeros_like(rows), torch.ones_like(scales), torch.zeros_like(norms)
    lab = [torch.zeros(40, 2, device=DEV) for _ in range(2)]
    rb.rb_bank_replace(torch.arange(40, dtype=torch.int32, device=DEV), x, lab[0], lab[1], z[0],
                       z[2], lab[0].clone(), lab[1].clone(), scales=z[1])
    assert torch.equal(z[0], rows) and torch.equal(z[1], scales) and torch.equal(z[2], norms)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_turnover(dtype):
    """A bank in use: predict and assign, accumulate, evict, replace, predict again."""
    import paper_2606_17949_amd as rb
    import synth
    cfg = synth.CONFIGS["tiny"]
    B, N, d, M = cfg.B, 1500, 96, cfg.M
    g = torch.Generator(device=DEV).manual_seed(3)
    src = torch.float32 if dtype == "f32" else torch.bfloat16

    def rows(n):
        x = torch.randn(n, d, generator=g, device=DEV)
        return (x / x.norm(dim=1, keepdim=True)).to(src)
    bank, scales = rows(N), None
    if dtype == "q4":
        bank, scales, norms = rb.rb_bank_pack(bank)
    else:
        norms = rb.rb_bank_norms(bank)
    qual = torch.rand(N, M, generator=g, device=DEV)
    ln = 1.0 + 300.0 * torch.rand(N, M, generator=g, device=DEV)
    mask = torch.ones(N, dtype=torch.uint8, device=DEV)
    usage = torch.zeros(N, device=DEV)
    inst = rb.DeviceInstances.from_host(synth.make_instances(cfg), DEV)
    plen = torch.from_numpy(synth.make_prompt_lens(cfg)).to(DEV)
    # every other row may go; the 25 new ones are the next batch's own prompts
    may_go = (torch.arange(N, device=DEV) % 2).to(torch.uint8)
    for step in range(3):
        q = rows(B)
        q_hat, l_hat, lse = rb.rb_attend(q, bank, norms, 6.0, qual, ln, scales=scales,
                                         row_mask=mask)
        assign = rb.rb_assign(q_hat, l_hat, plen, inst, cfg.weights)[0]
        rb.rb_attend_usage(q, bank, norms, 6.0, lse, usage, decay=0.9, scales=scales,
                           row_mask=mask)
        new = torch.cat((q, rows(9)))
        n = new.shape[0]
        before = usage.cpu().numpy()
        at = rb.rb_bank_evict(usage, n, may_go=may_go)
        nq = torch.ones(n, M, device=DEV)
        nl = torch.full((n, M), 77.0, device=DEV)
        rb.rb_bank_replace(at, new, nq, nl, bank, norms, qual, ln, scales=scales, usage=usage,
                           usage0=0.01)
        torch.cuda.synchronize()
        assert ((assign >= 0) & (assign < inst.I)).all()
        assert np.array_equal(at.cpu().numpy(), victims_of(before, may_go.cpu().numpy(), n))
        assert (qual[at.long()] == 1.0).all() and (usage[at.long()] == 0.01).all()
        # requests that are in the bank now, asked sharply, get their own labels
        # (a row held in 4 bits is some way off its request: only nearly)
        q_hat, l_hat, _ = rb.rb_attend(q, bank, norms, 400.0, qual, ln, scales=scales,
                                       row_mask=mask)
        x = ref.unpack4(bank, scales) if scales is not None else bank.double()
        for k, (value, bound) in ref.attend(q, x, 400.0, qual, ln, mask).items():
            if k != "lse":
                ref.check(k, q_hat if k == "q_hat" else l_hat, value, bound)
        if scales is None:
            assert (q_hat - 1.0).abs().max() < 1e-4 and (l_hat - 77.0).abs().max() < 0.01
