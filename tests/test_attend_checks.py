"""What the attention and bank-row calls refuse (no GPU needed): on the host,
before any device work."""
import ctypes
import math

import pytest
import torch

import paper_2606_17949_amd as rb

L = rb._lib
FAKE = ctypes.c_void_p(0x10000)        # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10004)


def attend(q=FAKE, x=FAKE, sc=None, norms=FAKE, dt=rb.RB_BF16, B=4, N=100, d=64, beta=1.0,
           mask=None, qual=FAKE, ln=FAKE, M=3, qh=FAKE, lh=FAKE, lse=FAKE, ws=FAKE, n=1 << 40):
    return L.rb_attend(q, x, sc, norms, dt, B, N, d, beta, mask, qual, ln, M, qh, lh, lse, ws, n,
                       None)


def backward(q=FAKE, x=FAKE, norms=FAKE, dt=rb.RB_BF16, B=4, N=100, d=64, beta=1.0, mask=None,
             qual=FAKE, ln=FAKE, M=3, qh=FAKE, lh=FAKE, lse=FAKE, dq=FAKE, dl=FAKE, dlse=None,
             o1=FAKE, o2=FAKE, o3=FAKE, o4=FAKE, o5=FAKE, ws=FAKE, n=1 << 40):
    return L.rb_attend_backward(q, x, norms, dt, B, N, d, beta, mask, qual, ln, M, qh, lh, lse, dq,
                                dl, dlse, o1, o2, o3, o4, o5, ws, n, None)


def usage(q=FAKE, x=FAKE, sc=None, norms=FAKE, dt=rb.RB_BF16, B=4, N=100, d=64, beta=1.0,
          mask=None, lse=FAKE, decay=0.5, use=FAKE, ws=FAKE, n=1 << 40):
    return L.rb_attend_usage(q, x, sc, norms, dt, B, N, d, beta, mask, lse, decay, use, ws, n, None)


SIZES = [(dict(B=-1), rb.RB_ERR_DIMS), (dict(N=0), rb.RB_ERR_DIMS), (dict(d=0), rb.RB_ERR_DIMS),
         (dict(B=1 << 23), rb.RB_ERR_DIMS),
         (dict(d=60), rb.RB_ERR_DIMS), (dict(d=2056), rb.RB_ERR_DIMS),
         (dict(dt=rb.RB_F32, d=6), rb.RB_ERR_DIMS), (dict(dt=7), rb.RB_ERR_DTYPE),
         (dict(dt=-1), rb.RB_ERR_DTYPE), (dict(beta=0.0), rb.RB_ERR_VALUE),
         (dict(beta=-1.0), rb.RB_ERR_VALUE), (dict(beta=math.nan), rb.RB_ERR_VALUE),
         (dict(beta=math.inf), rb.RB_ERR_VALUE), (dict(beta=2e30), rb.RB_ERR_VALUE),
         (dict(q=None), rb.RB_ERR_NULL), (dict(x=None), rb.RB_ERR_NULL),
         (dict(norms=None), rb.RB_ERR_NULL), (dict(q=ODD), rb.RB_ERR_ALIGN),
         (dict(x=ODD), rb.RB_ERR_ALIGN)]


@pytest.mark.parametrize("kw,code", SIZES)
@pytest.mark.parametrize("call", [attend, backward, usage])
def test_shared_refusals(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("call", [attend, usage])
@pytest.mark.parametrize("kw,code", [(dict(d=40), rb.RB_ERR_DIMS), (dict(sc=None), rb.RB_ERR_NULL)])
def test_4_bit_refusals(call, kw, code):
    assert call(**{"dt": rb.RB_Q4, "sc": FAKE, **kw}) == code


@pytest.mark.parametrize("call", [attend, backward])
@pytest.mark.parametrize("kw,code", [
    (dict(M=0), rb.RB_ERR_DIMS), (dict(M=rb.RB_MAX_M + 1), rb.RB_ERR_DIMS),
    (dict(qual=None), rb.RB_ERR_NULL), (dict(ln=None), rb.RB_ERR_NULL),
    (dict(qh=None), rb.RB_ERR_NULL), (dict(lh=None), rb.RB_ERR_NULL)])
def test_label_refusals(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dt=rb.RB_Q4), rb.RB_ERR_DTYPE), (dict(lse=None), rb.RB_ERR_NULL),
    (dict(dq=None), rb.RB_ERR_NULL), (dict(dl=None), rb.RB_ERR_NULL),
    (dict(o1=ODD), rb.RB_ERR_ALIGN), (dict(o2=ODD), rb.RB_ERR_ALIGN)])
def test_backward_refusals(kw, code):
    assert backward(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(decay=-0.1), rb.RB_ERR_VALUE), (dict(decay=1.5), rb.RB_ERR_VALUE),
    (dict(decay=math.nan), rb.RB_ERR_VALUE), (dict(use=None), rb.RB_ERR_NULL),
    (dict(lse=None), rb.RB_ERR_NULL)])
def test_usage_refusals(kw, code):
    assert usage(**kw) == code


def test_empty_batch_needs_no_pointers():
    assert attend(B=0, q=None, x=None, ws=None, n=0) == rb.RB_OK


def test_workspace_size_refusals():
    n = ctypes.c_size_t(0)
    p = ctypes.byref(n)
    assert L.rb_attend_workspace_size(4, 100, 64, rb.RB_BF16, 3, None) == rb.RB_ERR_NULL
    assert L.rb_attend_workspace_size(4, 100, 60, rb.RB_BF16, 3, p) == rb.RB_ERR_DIMS
    assert L.rb_attend_workspace_size(4, 100, 64, rb.RB_BF16, 0, p) == rb.RB_ERR_DIMS
    assert L.rb_attend_workspace_size(4, 100, 64, 9, 3, p) == rb.RB_ERR_DTYPE
    assert L.rb_attend_backward_workspace_size(4, 100, 64, rb.RB_Q4, 3, p) == rb.RB_ERR_DTYPE
    assert L.rb_attend_backward_workspace_size(4, 0, 64, rb.RB_F32, 3, p) == rb.RB_ERR_DIMS
    assert L.rb_attend_usage_workspace_size(-1, 100, 64, rb.RB_F32, p) == rb.RB_ERR_DIMS
    assert L.rb_evict_workspace_size(0, p) == rb.RB_ERR_DIMS
    assert L.rb_evict_workspace_size(5, None) == rb.RB_ERR_NULL
    for B0 in (L.rb_attend_workspace_size, L.rb_attend_backward_workspace_size):
        assert B0(0, 100, 64, rb.RB_F32, 3, p) == rb.RB_OK and n.value == 0


@pytest.mark.parametrize("dt,N,d,x,rows,code", [
    (rb.RB_Q4, 4, 64, FAKE, FAKE, rb.RB_ERR_DTYPE), (rb.RB_F32, 4, 48, FAKE, FAKE, rb.RB_ERR_DIMS),
    (rb.RB_F32, 0, 64, FAKE, FAKE, rb.RB_ERR_DIMS), (rb.RB_F32, 4, 64, None, FAKE, rb.RB_ERR_NULL),
    (rb.RB_F32, 4, 64, ODD, FAKE, rb.RB_ERR_ALIGN), (rb.RB_F32, 4, 64, FAKE, ODD, rb.RB_ERR_ALIGN)])
def test_pack_refusals(dt, N, d, x, rows, code):
    assert L.rb_bank_pack(x, dt, N, d, rows, FAKE, FAKE, None) == code


@pytest.mark.parametrize("N,n,u,v,ws,size,code", [
    (0, 0, FAKE, FAKE, FAKE, 1 << 30, rb.RB_ERR_DIMS), (5, 6, FAKE, FAKE, FAKE, 1 << 30, rb.RB_ERR_DIMS),
    (5, -1, FAKE, FAKE, FAKE, 1 << 30, rb.RB_ERR_DIMS), (5, 2, None, FAKE, FAKE, 1 << 30, rb.RB_ERR_NULL),
    (5, 2, FAKE, None, FAKE, 1 << 30, rb.RB_ERR_NULL), (5, 2, FAKE, FAKE, None, 1 << 30, rb.RB_ERR_WORKSPACE),
    (5, 2, FAKE, FAKE, FAKE, 64, rb.RB_ERR_WORKSPACE), (5, 2, FAKE, FAKE, ODD, 1 << 30, rb.RB_ERR_ALIGN),
    (5, 0, None, None, None, 0, rb.RB_OK)])
def test_evict_refusals(N, n, u, v, ws, size, code):
    assert L.rb_bank_evict(u, None, N, n, v, ws, size, None) == code


def replace(at=FAKE, n=3, new=FAKE, src=rb.RB_BF16, nq=FAKE, nl=FAKE, M=2, x=FAKE, sc=None,
            norms=FAKE, dt=rb.RB_BF16, N=9, d=64, qual=FAKE, ln=FAKE, use=None, u0=0.0):
    return L.rb_bank_replace(at, n, new, src, nq, nl, M, x, sc, norms, dt, N, d, qual, ln, use, u0,
                             None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), rb.RB_ERR_DIMS), (dict(N=0), rb.RB_ERR_DIMS), (dict(d=20), rb.RB_ERR_DIMS),
    (dict(dt=rb.RB_Q4, sc=FAKE, d=40), rb.RB_ERR_DIMS), (dict(M=0), rb.RB_ERR_DIMS),
    (dict(src=rb.RB_F32), rb.RB_ERR_DTYPE), (dict(dt=rb.RB_Q4, sc=FAKE, src=rb.RB_Q4), rb.RB_ERR_DTYPE),
    (dict(dt=5), rb.RB_ERR_DTYPE), (dict(u0=math.nan), rb.RB_ERR_VALUE), (dict(at=None), rb.RB_ERR_NULL),
    (dict(new=None), rb.RB_ERR_NULL), (dict(nq=None), rb.RB_ERR_NULL), (dict(x=None), rb.RB_ERR_NULL),
    (dict(norms=None), rb.RB_ERR_NULL), (dict(ln=None), rb.RB_ERR_NULL),
    (dict(dt=rb.RB_Q4, sc=None), rb.RB_ERR_NULL), (dict(new=ODD), rb.RB_ERR_ALIGN),
    (dict(x=ODD), rb.RB_ERR_ALIGN), (dict(n=0, at=None), rb.RB_OK)])
def test_replace_refusals(kw, code):
    assert replace(**kw) == code


def test_header_knows_the_new_names():
    import os
    text = open(os.path.join(os.path.dirname(rb.LIB_PATH), "..", "include",
                             "routebalance.h")).read()
    assert "RB_Q4 = 2" in text and "RB_ERR_VALUE = -10" in text
    assert rb.rb_status_string(rb.RB_ERR_VALUE).startswith("RB_ERR_VALUE")


# ------------------------------------------------------------------ the binding

B, N, d, M = 4, 50, 64, 3


def good(dtype=torch.bfloat16):
    return dict(q=torch.zeros(B, d, dtype=dtype), x=torch.zeros(N, d, dtype=dtype),
                norms=torch.zeros(N), qual=torch.zeros(N, M), ln=torch.zeros(N, M),
                bm=torch.zeros(B, M), b=torch.zeros(B))


def raises(name, fn, *a, **kw):
    with pytest.raises(ValueError, match=name):
        fn(*a, **kw)


def test_binding_attend():
    g = good()
    args = [g["q"], g["x"], g["norms"], 1.0, g["qual"], g["ln"]]

    def with_(i, v):
        a = list(args)
        a[i] = v
        return a
    raises("queries", rb.rb_attend, *with_(0, g["q"].float()))
    raises("queries", rb.rb_attend, *with_(0, g["q"][:, :32].contiguous()))
    raises("bank", rb.rb_attend, *with_(1, g["x"].double()))
    raises("bank_norms", rb.rb_attend, *with_(2, torch.zeros(N + 1)))
    raises("bank_len", rb.rb_attend, *with_(5, torch.zeros(N, M + 1)))
    raises("row_mask", rb.rb_attend, *args, row_mask=torch.zeros(N, dtype=torch.bool))
    raises("scales", rb.rb_attend, *args, scales=torch.zeros(N, 2, dtype=torch.uint8))
    raises("q_hat", rb.rb_attend, *args, q_hat=torch.zeros(B, M + 1))
    raises("lse", rb.rb_attend, *args, lse=torch.zeros(B, 1))
    raises("ws", rb.rb_attend, *args, ws=torch.zeros(9))
    x4 = torch.zeros(N, d // 2, dtype=torch.uint8)
    raises("scales", rb.rb_attend, *with_(1, x4))
    raises("scales", rb.rb_attend, *with_(1, x4), scales=torch.zeros(N, 3, dtype=torch.uint8))
    raises("GPU", rb.rb_attend, *args, ws=torch.zeros(256, dtype=torch.uint8))


def test_binding_backward_and_usage():
    g = good()
    args = [g["q"], g["x"], g["norms"], 1.0, g["qual"], g["ln"], g["bm"], g["bm"], g["b"], g["bm"],
            g["bm"]]
    raises("dl_hat", rb.rb_attend_backward, *args[:-1], torch.zeros(B, M + 1))
    raises("dlse", rb.rb_attend_backward, *args, dlse=torch.zeros(B + 1))
    raises("d_bank", rb.rb_attend_backward, *args, d_bank=torch.zeros(N, d))
    raises("d_qual", rb.rb_attend_backward, *args, d_qual=torch.zeros(N, M + 1))
    raises("usage", rb.rb_attend_usage, *args[:4], g["b"], torch.zeros(N - 1))
    raises("lse", rb.rb_attend_usage, *args[:4], torch.zeros(B + 1), torch.zeros(N))


def test_binding_rows():
    g = good()
    raises("32", rb.rb_bank_pack, torch.zeros(4, 48))
    raises("bank", rb.rb_bank_pack, torch.zeros(4, 64, dtype=torch.float16))
    raises("usage", rb.rb_bank_evict, torch.zeros(4, 4), 1)
    raises("may_go", rb.rb_bank_evict, torch.zeros(4), 1, may_go=torch.zeros(4))
    raises("victims", rb.rb_bank_evict, torch.zeros(4), 1,
           victims=torch.zeros(2, dtype=torch.int32))
    at = torch.zeros(2, dtype=torch.int32)
    args = [at, g["x"][:2], g["qual"][:2], g["ln"][:2], g["x"], g["norms"], g["qual"], g["ln"]]
    raises("at", rb.rb_bank_replace, at.long(), *args[1:])
    raises("new_rows", rb.rb_bank_replace, at, g["x"][:2].float(), *args[2:])
    raises("new_qual", rb.rb_bank_replace, at, g["x"][:2], g["qual"][:1], *args[3:])
    raises("usage", rb.rb_bank_replace, *args, usage=torch.zeros(N + 1))
