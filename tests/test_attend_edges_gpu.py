"""Attention over the bank at the edges of what its calls allow (GPU): label
counts past every table, views that start anywhere, workspaces of a larger
batch, other streams, two calls at once, captured calls, long banks."""
import math

import pytest
import torch

import attend_ref as ref
from test_attend_gpu import DEV, backward, dirty, forward, make

pytestmark = pytest.mark.gpu

CODES = {"f32": 0, "bf16": 1, "q4": 2}


def check_all(got, want, label=""):
    for k, (value, bound) in want.items():
        if k not in got:
            continue
        half = torch.finfo(got[k].dtype).eps / 2
        if got[k].dtype == torch.float32:
            half = 0.0
        print(k, ref.check(k, got[k], value, bound + half * value.abs() + ref.T, label), flush=True)


def gradients(s, beta, out):
    return ref.backward(s["queries"], s["x"], beta, s["qual"], s["len"], out["q_hat"],
                        out["l_hat"], out["lse"], s["dq_hat"], s["dl_hat"], s["dlse"], s["mask"])


@pytest.mark.parametrize("wanted", [None, ("d_queries",), ("d_qual", "d_len")])
@pytest.mark.parametrize("dtype,B,N,d,M", [
    # a tile's label gradients and its requests are more than a workgroup's LDS;
    # tiles of two groups of requests of which the batch has three or one
    ("bf16", 40, 300, 64, 1024), ("bf16", 3, 100, 2048, 1024), ("bf16", 17, 65, 2048, 300),
    ("f32", 20, 300, 2048, 1024), ("f32", 1, 33, 2048, 700)])
def test_many_labels(dtype, B, N, d, M, wanted):
    import paper_2606_17949_amd as rb
    s = make(dtype, B, N, d, M, seed=M, mask="some")
    out = forward(s, 4.0, ws=dirty(rb.rb_attend_workspace_size(B, N, d, CODES[dtype], M)))
    check_all(out, ref.attend(s["queries"], s["x"], 4.0, s["qual"], s["len"], s["mask"]))
    kw = {}
    if wanted:
        shape = {"d_queries": (B, d), "d_qual": (N, M), "d_len": (N, M)}
        kw = {k: torch.empty(shape[k], device=DEV,
                             dtype=s["queries"].dtype if k == "d_queries" else torch.float32)
              for k in wanted}
    got = backward(s, 4.0, out, ws=dirty(
        rb.rb_attend_backward_workspace_size(B, N, d, CODES[dtype], M)), **kw)
    torch.cuda.synchronize()
    check_all(got, gradients(s, 4.0, out))


@pytest.mark.parametrize("dtype,N,d", [("f32", 500, 32), ("f32", 60_000, 96), ("bf16", 500, 64),
                                       ("bf16", 60_000, 128), ("q4", 500, 64), ("q4", 60_000, 32),
                                       ("bf16", 3, 768), ("f32", 7, 2048), ("bf16", 2_000_000, 16)])
def test_workspace_of_a_larger_batch(dtype, N, d):
    """The size asked for grows with the batch, so that one workspace serves all."""
    import paper_2606_17949_amd as rb
    sizes = [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 192, 255, 256, 257,
             300, 384, 500, 512, 513, 777, 1024, 1300, 2048, 4000, 5001, 9000, 20_000, 70_000]
    calls = [lambda b: rb.rb_attend_workspace_size(b, N, d, CODES[dtype], 4),
             lambda b: rb.rb_attend_workspace_size(b, N, d, CODES[dtype], 20),
             lambda b: rb.rb_attend_usage_workspace_size(b, N, d, CODES[dtype])]
    if dtype != "q4":
        calls.append(lambda b: rb.rb_attend_backward_workspace_size(b, N, d, CODES[dtype], 4))
    for call in calls:
        asked = [call(b) for b in sizes]
        assert asked == sorted(asked)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_smaller_batches_in_one_workspace(dtype):
    import paper_2606_17949_amd as rb
    B, N, d, M = 300, 20_000, 128, 4
    s = make(dtype, B, N, d, M, mask="some")
    ws = dirty(rb.rb_attend_workspace_size(B, N, d, CODES[dtype], M))
    uws = dirty(rb.rb_attend_usage_workspace_size(B, N, d, CODES[dtype]))
    gws = None if dtype == "q4" else dirty(
        rb.rb_attend_backward_workspace_size(B, N, d, CODES[dtype], M))
    for b in (1, 16, 17, 64, 130, 256, 300):
        part = {k: v[:b] if k in ("queries", "dq_hat", "dl_hat", "dlse") else v
                for k, v in s.items()}
        for w in (ws, uws, gws):
            if w is not None:
                w.fill_(0xff)
        one, two = forward(part, 6.0, ws=ws), forward(part, 6.0)
        for k in one:
            assert torch.equal(one[k], two[k]), (b, k)
        use = torch.zeros(2, N, device=DEV)
        for u, w in zip(use, (uws, None)):
            rb.rb_attend_usage(part["queries"], s["bank"], s["norms"], 6.0, one["lse"], u,
                               scales=s["scales"], row_mask=s["mask"], ws=w)
        assert torch.equal(use[0], use[1]), b
        if dtype != "q4":
            one, two = backward(part, 6.0, one, ws=gws), backward(part, 6.0, one)
            for k in one:
                assert torch.equal(one[k], two[k]), (b, k)


def moved(t, by):
    """The same values in a view that starts `by` elements into its storage."""
    if t is None:
        return None
    buf = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    v = buf[by:].view(t.shape)
    v.copy_(t)
    return v


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("B,N,d,M", [(5, 333, 64, 3), (300, 20_011, 128, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_views_that_start_anywhere(dtype, B, N, d, M, by):
    """Norms, masks, labels, scales and all fp32 results need no alignment but
    their elements' own: the same bits at every place."""
    import paper_2606_17949_amd as rb
    s = make(dtype, B, N, d, M, mask="some")
    t = dict(s)
    for k in ("norms", "mask", "qual", "len", "scales", "dq_hat", "dl_hat", "dlse"):
        t[k] = moved(s[k], by)
    out = forward(s, 5.0)
    place = {k: moved(torch.zeros_like(v), by) for k, v in out.items()}
    forward(t, 5.0, **place)
    for k in out:
        assert torch.equal(out[k], place[k]), k
    use = torch.rand(N, device=DEV)
    use2 = moved(use, by)
    for x, o, u in ((s, out, use), (t, place, use2)):
        rb.rb_attend_usage(x["queries"], x["bank"], x["norms"], 5.0, o["lse"], u, decay=0.5,
                           scales=x["scales"], row_mask=x["mask"])
    assert torch.equal(use, use2)
    want = rb.rb_bank_evict(use, 17, may_go=s["mask"])
    got = moved(torch.zeros_like(want), by)
    rb.rb_bank_evict(use2, 17, may_go=t["mask"], victims=got)
    assert torch.equal(want, got)
    if dtype == "q4":
        return
    whole = backward(s, 5.0, out)
    kw = {k: torch.empty_like(v) if k in ("d_queries", "d_bank") else
          moved(torch.zeros_like(v), by) for k, v in whole.items()}
    backward(t, 5.0, place, **kw)
    for k in whole:
        assert torch.equal(whole[k], kw[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_two_streams_at_once(dtype):
    """Calls on two streams, each with what it needs made by the call itself."""
    import paper_2606_17949_amd as rb
    sets = [make(dtype, 70, 30_000, 128, 4, seed=i, mask="some") for i in range(2)]

    def run(s, stream=None):
        out = forward(s, 5.0, stream=stream)
        use = torch.zeros(30_000, device=DEV) if stream is None else s["use"]
        rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], 5.0, out["lse"], use,
                           scales=s["scales"], row_mask=s["mask"], stream=stream)
        at = rb.rb_bank_evict(use, 99, stream=stream)
        grads = {} if dtype == "q4" else backward(s, 5.0, out, stream=stream)
        return {**out, **grads, "usage": use, "at": at}
    want = [run(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for s in sets:
            s["use"] = torch.zeros(30_000, device=DEV)
        torch.cuda.synchronize()
        got = []
        for s, st in zip(sets, streams):
            got.append(run(s, st))
            # memory that the call let go of is not the current stream's to take
            torch.empty(64 << 20, dtype=torch.uint8, device=DEV).fill_(0xff)
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            for k in w:
                assert torch.equal(w[k], g[k]), k


def test_another_devices_stream_is_refused():
    import paper_2606_17949_amd as rb
    s = make("bf16", 2, 20, 32, 2)

    class Other:
        device = torch.device("cuda", 7)
        cuda_stream = 0
    with pytest.raises(ValueError, match="stream"):
        forward(s, 1.0, stream=Other())


@pytest.mark.parametrize("B,N,d", [(1, 14_000, 96), (40, 14_000, 96), (300, 20_011, 128)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "q4"])
def test_turnover_captured(dtype, B, N, d):
    """Predict, accumulate, take gradients, evict and replace in one graph: each
    replay, with eager work between, does what the eager calls do."""
    import paper_2606_17949_amd as rb
    M, n = 4, 33
    s = make(dtype, B, N, d, M)
    g = torch.Generator(device=DEV).manual_seed(4)
    new = torch.randn(n, d, generator=g, device=DEV)
    new = (new / new.norm(dim=1, keepdim=True)).to(s["queries"].dtype)
    lab = torch.rand(2, n, M, generator=g, device=DEV)
    state = {"bank": s["bank"], "norms": s["norms"], "qual": s["qual"], "len": s["len"],
             "usage": torch.rand(N, generator=g, device=DEV)}
    if dtype == "q4":
        state["scales"] = s["scales"]
    first = {k: v.clone() for k, v in state.items()}
    code = CODES[dtype]
    ws = rb.attend_workspace(B, N, d, code, M)
    uws, ews = rb.attend_usage_workspace(B, N, d, code), rb.evict_workspace(N)
    out = {"q_hat": torch.empty(B, M, device=DEV), "l_hat": torch.empty(B, M, device=DEV),
           "lse": torch.empty(B, device=DEV)}
    at = torch.empty(n, dtype=torch.int32, device=DEV)
    grads, gws = {}, None
    if dtype != "q4":
        gws = rb.attend_backward_workspace(B, N, d, code, M)
        grads = {"d_queries": torch.empty_like(s["queries"]), "d_bank": torch.empty_like(s["bank"]),
                 "d_qual": torch.empty(N, M, device=DEV), "d_len": torch.empty(N, M, device=DEV),
                 "d_beta": torch.empty(B, device=DEV)}

    def step():
        forward(s, 5.0, ws=ws, **out)
        rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], 5.0, out["lse"], state["usage"],
                           decay=0.5, scales=s["scales"], ws=uws)
        if grads:
            backward(s, 5.0, out, ws=gws, **grads)
        rb.rb_bank_evict(state["usage"], n, victims=at, ws=ews)
        rb.rb_bank_replace(at, new, lab[0], lab[1], s["bank"], s["norms"], s["qual"], s["len"],
                           scales=s["scales"], usage=state["usage"], usage0=0.3)

    def reset():
        for k, v in first.items():
            state[k].copy_(v)
    seen = {**state, **out, **grads, "at": at}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    want = []
    reset()
    for _ in range(3):
        step()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in seen.items()})
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    reset()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for k in w:
            assert torch.equal(w[k], seen[k]), k
        forward(s, 2.0)   # (eager work between)
        torch.cuda.synchronize()


@pytest.mark.parametrize("B,N", [(3, 500), (40, 5000), (300, 20_011)])
def test_masked_4_bit_rows_hold_anything(B, N):
    """Scales and codes of masked rows that stand for no number change nothing."""
    import paper_2606_17949_amd as rb
    s = make("q4", B, N, 64, 3, mask="some")
    dead = s["mask"] == 0
    s["scales"][dead], s["bank"][dead] = 127, 0
    s["norms"][dead], s["qual"][dead], s["len"][dead] = 0.0, 0.0, 0.0
    out = forward(s, 5.0)
    use = torch.zeros(2, N, device=DEV)
    rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], 5.0, out["lse"], use[0],
                       scales=s["scales"], row_mask=s["mask"])
    s["scales"][dead] = torch.randint(0, 256, s["scales"][dead].shape, device=DEV,
                                      dtype=torch.uint8)
    s["scales"][dead, 0] = 255
    s["bank"][dead] = torch.randint(0, 256, s["bank"][dead].shape, device=DEV, dtype=torch.uint8)
    s["norms"][dead], s["qual"][dead], s["len"][dead] = math.inf, -math.inf, math.nan
    again = forward(s, 5.0)
    rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], 5.0, again["lse"], use[1],
                       scales=s["scales"], row_mask=s["mask"])
    for k in out:
        assert torch.equal(out[k], again[k]), k
    assert torch.equal(use[0], use[1])


@pytest.mark.parametrize("mask", [None, "some"])
@pytest.mark.parametrize("dtype,B,N,d", [("bf16", 513, 150_011, 32), ("f32", 200, 190_000, 20)])
def test_gradients_in_parts(dtype, B, N, d, mask):
    """Banks whose scores' gradients go by in several parts."""
    s = make(dtype, B, N, d, 2, mask=mask)
    out = forward(s, 5.0)
    got = backward(s, 5.0, out)
    torch.cuda.synchronize()
    check_all(got, gradients(s, 5.0, out))


@pytest.mark.parametrize("dtype,N,d,M", [("f32", 1_450_001, 768, 2), ("bf16", 2_900_001, 768, 2),
                                         ("q4", 11_400_001, 768, 1), ("bf16", 1_200_001, 32, 1000)])
def test_past_4_gb(dtype, N, d, M):
    """Rows (or labels) past 4 GB: a few live ones there and before, all others masked."""
    import paper_2606_17949_amd as rb
    g = torch.Generator(device=DEV).manual_seed(N)
    rows = torch.cat((torch.arange(0, 300, device=DEV),
                      torch.randint(0, N, (900,), generator=g, device=DEV),
                      torch.arange(N - 400, N, device=DEV))).unique()
    n = rows.numel()
    part = make(dtype, 3, n, d, M)
    s = dict(part)
    s["bank"] = torch.zeros(N, part["bank"].shape[1], dtype=part["bank"].dtype, device=DEV)
    s["bank"][rows] = part["bank"]
    if dtype == "q4":
        s["scales"] = torch.full((N, d // 32), 255, dtype=torch.uint8, device=DEV)
        s["scales"][rows] = part["scales"]
    s["mask"] = torch.zeros(N, dtype=torch.uint8, device=DEV)
    s["mask"][rows] = 1
    for k in ("norms", "qual", "len"):
        s[k] = torch.full((N,) + tuple(part[k].shape[1:]), math.nan, device=DEV)
        s[k][rows] = part[k]
    out = forward(s, 5.0)
    want = ref.attend(part["queries"], part["x"], 5.0, part["qual"], part["len"])
    check_all(out, want)
    use = torch.full((N,), 0.5, device=DEV)
    rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], 5.0, out["lse"], use, decay=0.5,
                       scales=s["scales"], row_mask=s["mask"])
    value, bound = ref.usage(part["queries"], part["x"], 5.0, out["lse"],
                             torch.full((n,), 0.5, device=DEV), 0.5)
    ref.check("usage", use[rows], value, bound)
    use[rows] = 0.25
    assert (use == 0.25).all()
    if dtype == "q4":
        return
    got = backward(s, 5.0, out)
    torch.cuda.synchronize()
    few = {k: v[rows] if k in ("d_bank", "d_qual", "d_len") else v for k, v in got.items()}
    check_all(few, gradients(part, 5.0, out))
    for k in ("d_bank", "d_qual", "d_len"):
        got[k][rows] = 0
        assert torch.count_nonzero(got[k]) == 0, k
