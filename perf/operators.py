"""Attention of requests over the labelled bank, its gradients, the bank held in
4 bits and the turnover of its rows, as cases that can be timed and checked.

A request b weighs every bank row n by a softmax over the negated squared
distances, with a sharpness beta:

    p[b][n] = exp(-beta * |q_b - x_n|^2) / sum over the unmasked rows j of exp(-beta * |q_b - x_j|^2)

Kinds of pass:
  attend    the predictions q_hat, l_hat (the labels' averages under p) and the
            logarithm of the denominator, over a bank of fp32, bf16 or 4-bit rows
  backward  the gradients of those three outputs: requests, bank rows, labels, beta
  usage     a bank row's accumulated weight: usage = decay * usage + sum over b of p[b]
  evict     the rows of least usage make room, and new rows take their places

4-bit rows: 32 elements share a scale 2^(s - 127); an element is one of 0, 0.5,
1, 1.5, 2, 3, 4, 6 (codes 0 to 7) times it, negated where bit 3 is set; a byte
holds two elements, the even one in its low half.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

_DEFAULTS = {"kind": "attend", "dtype": "bf16", "B": 64, "N": 100_000, "d": 768, "M": 4,
             "beta": 8.0, "mask": False, "decay": 0.9, "n": 0}


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one request over a bank of 14,919 prompts (384-d fp32 embeddings): the
        # latency of a router that decides every request by itself
        _case(name="attend_one", dtype="f32", B=1, N=14_919, d=384),
        # the online batch of 64 requests over 100,000 prompts
        _case(name="attend_online", B=64, N=100_000, d=768),
        # the high-load batch over a bank of HBM scale
        _case(name="attend_highload", B=256, N=1_000_000, d=768, beta=16.0),
        # one request over a 4-bit bank, some of its rows not labelled yet
        _case(name="attend4_one", dtype="q4", B=1, N=100_000, d=768, mask=True),
        # a small batch over a 4-bit bank of HBM scale
        _case(name="attend4_stream", dtype="q4", B=64, N=1_000_000, d=768),
        # fine-tuning the encoder and the labels over the 14,919-prompt bank, odd batch
        _case(name="backward_small", kind="backward", dtype="f32", B=27, N=14_919, d=384),
        # a training step of the online bank, some rows held out
        _case(name="backward_online", kind="backward", B=256, N=100_000, d=768, mask=True),
        # a large training batch of longer embeddings and more models
        _case(name="backward_large", kind="backward", B=1_000, N=60_001, d=1_024, M=8, beta=4.0),
        # the weight that one batch gives the rows of the online bank
        _case(name="usage_online", kind="usage", B=64, N=100_000, d=768),
        # and of the high-load one
        _case(name="usage_highload", kind="usage", B=256, N=1_000_000, d=768, beta=16.0),
        # a few labelled prompts replace the least used rows of the online bank
        _case(name="evict_online", kind="evict", N=100_000, d=768, n=64, mask=True),
        # a day's labelled prompts replace rows of the largest bank
        _case(name="evict_bulk", kind="evict", N=4_000_000, d=384, n=50_000, M=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "backward", "backward", "usage", "evict"])
    dtype = rng.choice(["f32", "bf16", "bf16"] + (["q4", "q4"] if kind in ("attend", "usage")
                                                  else []))
    d = rng.choice({"f32": [96, 128, 256, 300, 384, 384, 512, 768, 1_024],
                    "bf16": [128, 200, 256, 384, 512, 640, 768, 768, 1_000, 1_024, 1_536, 2_048],
                    "q4": [128, 160, 256, 384, 512, 768, 768, 1_024, 1_536, 2_048]}[dtype])
    case = _case(kind=kind, dtype=dtype, d=d, B=_log_int(rng, 1, 1_024), M=rng.randint(1, 16),
                 beta=round(math.exp(rng.uniform(math.log(2.0), math.log(32.0))), 2),
                 mask=rng.random() < 0.4, decay=rng.choice([1.0, 0.99, 0.9, 0.5]))
    row = d * {"f32": 4.0, "bf16": 2.0, "q4": 17 / 32}[dtype]
    if kind == "evict":
        N = _log_int(rng, 1_000, min(4_000_000, int(3e9 / row)))
        case.update(B=0, N=N, n=_log_int(rng, 1, max(1, min(N // 4, 50_000))))
        return case
    # no dearer than the largest listed cases: 1.5 GB of bank, and their arithmetic
    flops = (4e10 if dtype == "f32" else 3.9e11) / (5.0 if kind == "backward" else 1.0)
    most = min((4e8 if kind == "backward" else 1.5e9) / row, flops / (2.0 * case["B"] * d))
    case["N"] = _log_int(rng, 500, max(501, min(1_000_000, int(most))))
    return case


# ------------------------------------------------------------------ inputs


def _gen(seed, role):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1_000_003 + role) & ((1 << 62) - 1))


def _embeddings(case, centres, rows, g):
    """Mixture draws around unit-norm centres (noise radius 0.3), normalised."""
    d = case["d"]
    out = torch.empty(rows, d, device=DEV,
                      dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
    for r0 in range(0, rows, 1 << 18):
        r1 = min(rows, r0 + (1 << 18))
        u = torch.randint(0, centres.shape[0], (r1 - r0,), generator=g, device=DEV)
        x = torch.randn(r1 - r0, d, generator=g, device=DEV).mul_(0.3 / math.sqrt(d))
        x += centres[u]
        x /= x.norm(dim=1, keepdim=True)
        out[r0:r1] = x
    return out


def _labels(n, M, g):
    """Qualities in [0, 1], output lengths ~ round(LogNormal(5, 0.6))."""
    qual = torch.rand(n, M, generator=g, device=DEV)
    z = torch.randn(n, M, generator=g, device=DEV)
    return qual, torch.exp(5.0 + 0.6 * z).round_().clamp_min_(1.0)


def _hold4(rows):
    """(codes, scales, norms) of rows held in 4 bits: the scale of 32 elements is
    the least power of two under which none passes 6, ties between two elements go
    to the even code."""
    N, d = rows.shape
    codes = torch.empty(N, d // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(N, d // 32, dtype=torch.uint8, device=DEV)
    norms = torch.empty(N, device=DEV)
    for r0 in range(0, N, 1 << 17):
        x = rows[r0:r0 + (1 << 17)].float().view(-1, d // 32, 32)
        top = x.abs().amax(2)
        m, e = torch.frexp(top / 6.0)
        e = torch.where(m == 0.5, e - 1, e).clamp(-126, 127)
        e = torch.where(top == 0, torch.full_like(e, -126), e)
        y = (x.double() * torch.exp2(-e.double())[..., None]).float()
        a = y.abs()
        # halves of a step up to 2, then steps of 1 and 2
        code = torch.where(a <= 2.0, torch.round(a * 2.0),
                           torch.where(a <= 4.0, torch.round(a) + 2.0, torch.round(a * 0.5) + 4.0))
        code = code.clamp_max(7.0).to(torch.uint8)
        value = torch.tensor(_MAGNITUDES, device=DEV)[code.long()] * torch.exp2(e.float())[..., None]
        code = (code | (torch.signbit(y).to(torch.uint8) << 3)).view(-1, d)
        codes[r0:r0 + (1 << 17)] = code[:, 0::2] | (code[:, 1::2] << 4)
        scales[r0:r0 + (1 << 17)] = (e + 127).to(torch.uint8)
        norms[r0:r0 + (1 << 17)] = value.view(-1, d).square().sum(1)
    return codes, scales, norms


def prepare(case, seed):
    B, N, M = case["B"], case["N"], case["M"]
    s = {"case": case, "scales": None, "mask": None}
    g = _gen(seed, 0)
    centres = torch.randn(max(32, min(1_024, N // 100)), case["d"], generator=g, device=DEV)
    centres /= centres.norm(dim=1, keepdim=True)
    s["bank"] = _embeddings(case, centres, N, _gen(seed, 1))
    if case["dtype"] == "q4":
        s["bank"], s["scales"], s["norms"] = _hold4(s["bank"])
    else:
        s["norms"] = torch.empty(N, device=DEV)
        for r0 in range(0, N, 1 << 18):
            s["norms"][r0:r0 + (1 << 18)] = s["bank"][r0:r0 + (1 << 18)].float().square().sum(1)
    s["queries"] = _embeddings(case, centres, B, _gen(seed, 2))
    s["qual"], s["len"] = _labels(N, M, _gen(seed, 3))
    g = _gen(seed, 4)
    if case["mask"]:
        # attend, backward and usage read the rows of mask 1; eviction may take them
        s["mask"] = (torch.rand(N, generator=g, device=DEV) < 0.8).to(torch.uint8)
    if case["kind"] == "backward":
        out = _exact_attend(s, torch.float64)
        s["q_hat"], s["l_hat"], s["lse"] = (out[k].float() for k in ("q_hat", "l_hat", "lse"))
        s["dq_hat"] = torch.randn(B, M, generator=g, device=DEV) / B
        s["dl_hat"] = torch.randn(B, M, generator=g, device=DEV) * (1e-3 / B)
        s["dlse"] = torch.randn(B, generator=g, device=DEV) * (0.1 / B)
    if case["kind"] == "usage":
        s["lse"] = _exact_attend(s, torch.float64)["lse"].float()
        s["usage"] = torch.rand(N, generator=g, device=DEV)
    if case["kind"] == "evict":
        # most rows were weighed by something, a tenth by nothing
        s["usage"] = -torch.log(1.0 - torch.rand(N, generator=g, device=DEV))
        s["usage"][torch.rand(N, generator=g, device=DEV) < 0.1] = 0.0
        s["new_rows"] = _embeddings(case, centres, case["n"], _gen(seed, 5))
        s["new_qual"], s["new_len"] = _labels(case["n"], M, _gen(seed, 6))
    if own:
        _places(s)
    return s


def _places(s):
    """The workspace and the outputs that a program keeps from call to call."""
    import paper_2606_17949_amd as rb
    case = s["case"]
    B, N, d, M, kind = (case[k] for k in ("B", "N", "d", "M", "kind"))
    code = {"f32": rb.RB_F32, "bf16": rb.RB_BF16, "q4": rb.RB_Q4}[case["dtype"]]
    if kind == "attend":
        s["ws"] = rb.attend_workspace(B, N, d, code, M, device=DEV)
        s["out"] = {"q_hat": torch.empty(B, M, device=DEV), "l_hat": torch.empty(B, M, device=DEV),
                    "lse": torch.empty(B, device=DEV)}
    elif kind == "backward":
        s["ws"] = rb.attend_backward_workspace(B, N, d, code, M, device=DEV)
        s["out"] = {"d_queries": torch.empty_like(s["queries"]),
                    "d_bank": torch.empty_like(s["bank"]),
                    "d_qual": torch.empty(N, M, device=DEV), "d_len": torch.empty(N, M, device=DEV),
                    "d_beta": torch.empty(B, device=DEV)}
    elif kind == "usage":
        s["ws"] = rb.attend_usage_workspace(B, N, d, code, device=DEV)
    else:
        s["ws"] = rb.evict_workspace(N, device=DEV)
        s["victims"] = torch.empty(case["n"], dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------ the passes


def _rows32(s):
    """The bank in 32 bits."""
    if s["case"]["dtype"] != "q4":
        return s["bank"].float()
    N, d = s["case"]["N"], s["case"]["d"]
    byte = s["bank"].to(torch.int32)
    code = torch.stack((byte & 15, byte >> 4), 2).view(N, d)
    value = torch.tensor(_MAGNITUDES + tuple(-v for v in _MAGNITUDES), device=DEV)[code]
    scale = torch.exp2(s["scales"].float() - 127.0)
    return (value.view(N, d // 32, 32) * scale[..., None]).view(N, d)


def _distances32(s, x):
    q = s["queries"].float()
    return q.square().sum(1, keepdim=True) + s["norms"] - 2.0 * (q @ x.t())


def _weights32(s, dist, lse):
    """p[B][N] from the distances and the logarithm of the denominator."""
    score = -s["case"]["beta"] * dist
    if s["mask"] is not None:
        score.masked_fill_(s["mask"] == 0, -math.inf)
    return torch.exp(score - lse[:, None])


def _plain_attend(s):
    score = -s["case"]["beta"] * _distances32(s, _rows32(s))
    if s["mask"] is not None:
        score.masked_fill_(s["mask"] == 0, -math.inf)
    top = score.amax(1, keepdim=True)
    w = torch.exp(score - top)
    total = w.sum(1, keepdim=True)
    v = torch.cat((s["qual"], s["len"]), 1)
    # up to a million rows: 2,048 at a time in 32 bits, those sums in 64
    B, N = w.shape
    even = N // 2_048 * 2_048
    parts = w[:, :even].reshape(B, -1, 2_048).transpose(0, 1) @ v[:even].view(-1, 2_048, v.shape[1])
    mean = (parts.double().sum(0) + w[:, even:] @ v[even:]) / total
    M = s["case"]["M"]
    return {"q_hat": mean[:, :M].float(), "l_hat": mean[:, M:].float(),
            "lse": (top + torch.log(total))[:, 0]}


def _plain_backward(s):
    beta, dt = s["case"]["beta"], s["queries"].dtype
    x, q = _rows32(s), s["queries"].float()
    dist = _distances32(s, x)
    p = _weights32(s, dist, s["lse"])
    dp = s["dq_hat"] @ s["qual"].t() + s["dl_hat"] @ s["len"].t()
    dp -= (s["dq_hat"] * s["q_hat"] + s["dl_hat"] * s["l_hat"]).sum(1, keepdim=True)
    ds = p * (dp + s["dlse"][:, None])
    return {"d_queries": (2.0 * beta * (ds @ x - ds.sum(1, keepdim=True) * q)).to(dt),
            "d_bank": (2.0 * beta * (ds.t() @ q - ds.sum(0)[:, None] * x)).to(dt),
            "d_qual": p.t() @ s["dq_hat"], "d_len": p.t() @ s["dl_hat"],
            "d_beta": -(ds * dist).sum(1)}


def _plain_usage(s):
    p = _weights32(s, _distances32(s, _rows32(s)), s["lse"])
    s["usage"].mul_(s["case"]["decay"]).add_(p.sum(0))
    return {"usage": s["usage"]}


def _plain_evict(s):
    n = s["case"]["n"]
    key = s["usage"]
    if s["mask"] is not None:
        key = torch.where(s["mask"] != 0, key, torch.full_like(key, math.inf))
    at = torch.sort(key, stable=True).indices[:n]   # equal usage: the lower row first
    at = torch.sort(at).values
    s["bank"][at] = s["new_rows"]
    s["norms"][at] = s["new_rows"].float().square().sum(1)
    s["qual"][at] = s["new_qual"]
    s["len"][at] = s["new_len"]
    s["usage"][at] = 0.0
    return {"victims": at.to(torch.int32), "bank": s["bank"], "norms": s["norms"],
            "qual": s["qual"], "len": s["len"], "usage": s["usage"]}


def _own_run(s):
    import paper_2606_17949_amd as rb
    case = s["case"]
    if case["kind"] == "attend":
        rb.rb_attend(s["queries"], s["bank"], s["norms"], case["beta"], s["qual"], s["len"],
                     scales=s["scales"], row_mask=s["mask"], ws=s["ws"], **s["out"])
        return s["out"]
    if case["kind"] == "backward":
        rb.rb_attend_backward(s["queries"], s["bank"], s["norms"], case["beta"], s["qual"],
                              s["len"], s["q_hat"], s["l_hat"], s["lse"], s["dq_hat"],
                              s["dl_hat"], dlse=s["dlse"], row_mask=s["mask"], ws=s["ws"],
                              **s["out"])
        return s["out"]
    if case["kind"] == "usage":
        rb.rb_attend_usage(s["queries"], s["bank"], s["norms"], case["beta"], s["lse"],
                           s["usage"], decay=case["decay"], scales=s["scales"],
                           row_mask=s["mask"], ws=s["ws"])
        return {"usage": s["usage"]}
    rb.rb_bank_evict(s["usage"], case["n"], may_go=s["mask"], victims=s["victims"], ws=s["ws"])
    rb.rb_bank_replace(s["victims"], s["new_rows"], s["new_qual"], s["new_len"], s["bank"],
                       s["norms"], s["qual"], s["len"], usage=s["usage"])
    return {"victims": s["victims"], "bank": s["bank"], "norms": s["norms"], "qual": s["qual"],
            "len": s["len"], "usage": s["usage"]}


def run(state):
    if own:
        return _own_run(state)
    return {"attend": _plain_attend, "backward": _plain_backward, "usage": _plain_usage,
            "evict": _plain_evict}[state["case"]["kind"]](state)


def work(case):
    B, N, d, M, n = (case[k] for k in ("B", "N", "d", "M", "n"))
    esz = 4 if case["dtype"] == "f32" else 2
    bank = N * (d // 2 + d // 32 if case["dtype"] == "q4" else d * esz)
    mask = N if case["mask"] else 0
    req, labels = B * d * esz, N * M * 8
    if case["kind"] == "attend":
        return {"bytes": bank + N * 4 + mask + labels + req + B * (M * 8 + 4),
                "flops": 2 * B * N * (d + 2 * M)}
    if case["kind"] == "backward":
        # the scores, both products of their gradient, the labels' two
        return {"bytes": 2 * (bank + labels + req) + N * 4 + mask + B * (M * 16 + 12),
                "flops": 6 * B * N * d + 8 * B * N * M}
    if case["kind"] == "usage":
        return {"bytes": bank + N * 12 + mask + req + B * 4, "flops": 2 * B * N * d}
    return {"bytes": N * 4 + mask + 2 * n * (d * esz + M * 8) + n * 12, "flops": N + 2 * n * d}


# ------------------------------------------------------------------ in 64 bits


def _exact_rows(s):
    case = s["case"]
    if case["dtype"] != "q4":
        return s["bank"].double()
    low = torch.remainder(s["bank"], 16).long()
    high = torch.div(s["bank"], 16, rounding_mode="floor").long()
    table = torch.tensor([(-1.0) ** (c // 8) * _MAGNITUDES[c % 8] for c in range(16)], device=DEV,
                         dtype=torch.float64)
    x = torch.empty(case["N"], case["d"], device=DEV, dtype=torch.float64)
    x[:, 0::2] = table[low]
    x[:, 1::2] = table[high]
    for j in range(case["d"] // 32):
        x[:, 32 * j:32 * j + 32] *= torch.pow(2.0, s["scales"][:, j].double() - 127.0)[:, None]
    return x


def _exact_parts(s):
    """(first row, rows in 64 bits, scores, distances) of the bank, some rows at a time."""
    case, q = s["case"], s["queries"].double()
    x = _exact_rows(s)
    step = max(1, 400_000_000 // max(1, max(case["B"], case["d"])))
    for r0 in range(0, case["N"], step):
        part = x[r0:r0 + step]
        dist = torch.square(q).sum(1)[:, None] + torch.square(part).sum(1)[None] \
            - 2.0 * torch.matmul(q, part.t())
        score = dist * -case["beta"]
        if s["mask"] is not None:
            score[:, s["mask"][r0:r0 + step] == 0] = -math.inf
        yield r0, part, score, dist


def _exact_attend(s, kind):
    case, lse = s["case"], None
    M = case["M"]
    for r0, part, score, _ in _exact_parts(s):
        here = torch.logsumexp(score, 1)
        n = part.shape[0]
        v = torch.cat((s["qual"][r0:r0 + n], s["len"][r0:r0 + n]), 1).double()
        mean = torch.softmax(score, 1) @ v
        if lse is None:
            lse, out = here, mean
        else:
            both = torch.logaddexp(lse, here)
            out = out * torch.exp(lse - both)[:, None] + mean * torch.exp(here - both)[:, None]
            lse = both
    return {"q_hat": out[:, :M].to(kind), "l_hat": out[:, M:].to(kind), "lse": lse.to(kind)}


def exact(case, seed):
    s = prepare(case, seed)
    kind, beta = case["kind"], case["beta"]
    if kind == "attend":
        return _exact_attend(s, torch.float64)
    if kind == "evict":
        usage, n = s["usage"].cpu(), case["n"]
        rows = torch.arange(case["N"])
        if s["mask"] is not None:
            rows = rows[s["mask"].cpu() != 0]
        least = torch.argsort(usage[rows].double(), stable=True)[:n]
        at = rows[least].sort().values.to(DEV)
        bank, norms, qual, length = (s[k].double() for k in ("bank", "norms", "qual", "len"))
        usage = s["usage"].double()
        bank[at] = s["new_rows"].double()
        norms[at] = s["new_rows"].double().pow(2).sum(1)
        qual[at], length[at], usage[at] = s["new_qual"].double(), s["new_len"].double(), 0.0
        return {"victims": at.to(torch.int32), "bank": bank, "norms": norms, "qual": qual,
                "len": length, "usage": usage}
    q, lse = s["queries"].double(), s["lse"].double()
    if kind == "usage":
        usage = s["usage"].double() * case["decay"]
        for r0, part, score, _ in _exact_parts(s):
            usage[r0:r0 + part.shape[0]] += torch.exp(score - lse[:, None]).sum(0)
        return {"usage": usage}
    do = torch.cat((s["dq_hat"], s["dl_hat"]), 1).double()
    o = torch.cat((s["q_hat"], s["l_hat"]), 1).double()
    shift = s["dlse"].double() - (do * o).sum(1)
    dq = torch.zeros_like(q)
    dx = torch.empty(case["N"], case["d"], device=DEV, dtype=torch.float64)
    dv = torch.empty(case["N"], 2 * case["M"], device=DEV, dtype=torch.float64)
    db = torch.zeros(case["B"], device=DEV, dtype=torch.float64)
    for r0, part, score, dist in _exact_parts(s):
        n = part.shape[0]
        p = torch.exp(score - lse[:, None])
        v = torch.cat((s["qual"][r0:r0 + n], s["len"][r0:r0 + n]), 1).double()
        g = p * (do @ v.t() + shift[:, None])
        # d score / d q = -2 beta (q - x), and the opposite for x
        dq += 2.0 * beta * (torch.matmul(g, part) - g.sum(1)[:, None] * q)
        dx[r0:r0 + n] = 2.0 * beta * (torch.matmul(g.t(), q) - g.sum(0)[:, None] * part)
        dv[r0:r0 + n] = torch.matmul(p.t(), do)
        db -= (g * dist).sum(1)
    return {"d_queries": dq, "d_bank": dx, "d_qual": dv[:, :case["M"]].contiguous(),
            "d_len": dv[:, case["M"]:].contiguous(), "d_beta": db}
