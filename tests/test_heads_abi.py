"""CPU-side checks of layer norm's and linear attention's entry points: refusals before anything is launched, workspace sizes,
the host struct's layout."""
import ctypes

import pytest

from paper_2505_03803_amd import binding as B

FAKE = 0x10000          # a non-null, 16-byte aligned address that is never dereferenced


def norm(**kw):
    a = dict(x=FAKE, dt=B.BF16, M=4, groups=1, n=64, xs=0, w=FAKE, b=FAKE, eps=1e-5, y=FAKE, ys=0, mean=None, rstd=None)
    a.update(kw)
    return B.lib().rwkvq_layer_norm(a["x"], a["dt"], a["M"], a["groups"], a["n"], a["xs"], a["w"], a["b"], a["eps"], a["y"], a["ys"],
                                    a["mean"], a["rstd"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), B.ERR_NULL), (dict(y=None), B.ERR_NULL), (dict(dt=3), B.ERR_UNSUPPORTED), (dict(dt=-1), B.ERR_UNSUPPORTED),
    (dict(M=0), B.ERR_SHAPE), (dict(groups=0), B.ERR_SHAPE), (dict(n=0), B.ERR_SHAPE), (dict(n=-5), B.ERR_SHAPE),
    (dict(groups=1 << 13, n=1 << 12), B.ERR_SHAPE), (dict(M=1 << 30, groups=4), B.ERR_SHAPE),
    (dict(xs=63), B.ERR_SHAPE), (dict(ys=63), B.ERR_SHAPE), (dict(xs=1 << 40), B.ERR_SHAPE), (dict(xs=-64), B.ERR_SHAPE),
    (dict(eps=0.0), B.ERR_UNSUPPORTED), (dict(eps=-1e-5), B.ERR_UNSUPPORTED), (dict(eps=float("nan")), B.ERR_UNSUPPORTED),
    (dict(eps=float("inf")), B.ERR_UNSUPPORTED), (dict(eps=1e-60), B.ERR_UNSUPPORTED),
    (dict(x=FAKE + 2), B.ERR_ALIGN), (dict(y=FAKE + 8), B.ERR_ALIGN), (dict(w=FAKE + 2), B.ERR_ALIGN), (dict(b=FAKE + 1), B.ERR_ALIGN),
    (dict(mean=FAKE + 3), B.ERR_ALIGN), (dict(rstd=FAKE + 2), B.ERR_ALIGN),
])
def test_norm_rejects(kw, status):
    assert norm(**kw) == status


def norm_backward(**kw):
    a = dict(dy=FAKE, dys=0, x=FAKE, xs=0, dt=B.F16, M=4, groups=2, n=32, w=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, dxs=0, dw=FAKE, db=FAKE,
             ws=FAKE)
    a.update(kw)
    return B.lib().rwkvq_layer_norm_backward(a["dy"], a["dys"], a["x"], a["xs"], a["dt"], a["M"], a["groups"], a["n"], a["w"], a["mean"],
                                             a["rstd"], a["dx"], a["dxs"], a["dw"], a["db"], a["ws"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), B.ERR_NULL), (dict(x=None), B.ERR_NULL), (dict(mean=None), B.ERR_NULL), (dict(rstd=None), B.ERR_NULL),
    (dict(ws=None), B.ERR_NULL), (dict(dw=None), B.ERR_NULL), (dict(db=None), B.ERR_NULL), (dict(dx=None, dw=None, db=None), B.ERR_NULL),
    (dict(dt=7), B.ERR_UNSUPPORTED), (dict(M=-1), B.ERR_SHAPE), (dict(n=0), B.ERR_SHAPE), (dict(dys=32), B.ERR_SHAPE),
    (dict(dxs=63), B.ERR_SHAPE), (dict(xs=1), B.ERR_SHAPE), (dict(dx=FAKE + 4), B.ERR_ALIGN), (dict(dy=FAKE + 2), B.ERR_ALIGN),
    (dict(ws=FAKE + 4), B.ERR_ALIGN), (dict(dw=FAKE + 2), B.ERR_ALIGN), (dict(mean=FAKE + 1), B.ERR_ALIGN),
])
def test_norm_backward_rejects(kw, status):
    assert norm_backward(**kw) == status


def heads(**kw):
    a = dict(n_seqs=2, n_tokens=10, n_heads=4, head_dim=64)
    a.update(kw)
    return B.Heads(a.pop("n_seqs"), a.pop("n_tokens"), a.pop("n_heads"), a.pop("head_dim"), **a)


HEADS = [
    (dict(n_seqs=0), B.ERR_SHAPE), (dict(n_tokens=0), B.ERR_SHAPE), (dict(n_heads=0), B.ERR_SHAPE), (dict(head_dim=0), B.ERR_SHAPE),
    (dict(head_dim=60), B.ERR_UNSUPPORTED), (dict(head_dim=136), B.ERR_UNSUPPORTED), (dict(n_tokens=11), B.ERR_SHAPE),
    (dict(r_stride=255), B.ERR_SHAPE), (dict(r_stride=260), B.ERR_ALIGN), (dict(k_stride=257), B.ERR_ALIGN), (dict(v_stride=-8), B.ERR_SHAPE),
    (dict(out_stride=248), B.ERR_SHAPE), (dict(out_stride=1 << 40), B.ERR_SHAPE), (dict(slots=FAKE), B.ERR_SHAPE),
    (dict(slots=FAKE + 2, n_slots=4), B.ERR_ALIGN), (dict(offsets=FAKE + 1), B.ERR_ALIGN),
    (dict(n_seqs=1, n_tokens=1 << 30, n_heads=64), B.ERR_SHAPE), (dict(n_heads=1 << 20), B.ERR_SHAPE),
]


def attention(h, **kw):
    a = dict(r=FAKE, k=FAKE, v=FAKE, dt=B.F16, w=FAKE, u=FAKE, s=FAKE, so=FAKE, out=FAKE, ws=FAKE)
    a.update(kw)
    return B.lib().rwkvq_linear_attention(h.ref if h else None, a["r"], a["k"], a["v"], a["dt"], a["w"], a["u"], a["s"], a["so"], a["out"],
                                          a["ws"], None)


def attention_backward(h, **kw):
    a = dict(r=FAKE, k=FAKE, v=FAKE, do=FAKE, dt=B.BF16, w=FAKE, u=FAKE, s=FAKE, ds=FAKE, dr=FAKE, dk=FAKE, dv=FAKE, dw=FAKE, du=FAKE, di=FAKE,
             ws=FAKE)
    a.update(kw)
    return B.lib().rwkvq_linear_attention_backward(h.ref if h else None, a["r"], a["k"], a["v"], a["do"], a["dt"], a["w"], a["u"], a["s"],
                                                   a["ds"], a["dr"], a["dk"], a["dv"], a["dw"], a["du"], a["di"], a["ws"], None)


@pytest.mark.parametrize("kw,status", HEADS)
def test_heads_rejects(kw, status):
    h = heads(**kw)
    assert attention(h) == status and attention_backward(h) == status
    assert B.rwkvq_linear_attention_workspace_size(h) == 0 and B.rwkvq_linear_attention_backward_workspace_size(h) == 0


@pytest.mark.parametrize("name", ["r", "k", "v", "w", "u", "out"])
def test_attention_rejects_null_and_unaligned(name):
    assert attention(heads(), **{name: None}) == B.ERR_NULL
    assert attention(heads(), **{name: FAKE + 2}) == B.ERR_ALIGN
    assert attention(None) == B.ERR_NULL and attention(heads(), dt=B.F32) == B.ERR_UNSUPPORTED
    assert attention(heads(), s=FAKE + 8) == B.ERR_ALIGN and attention(heads(), so=FAKE + 4) == B.ERR_ALIGN


@pytest.mark.parametrize("name", ["r", "k", "v", "do", "w", "u", "dr", "dk", "dv", "dw", "du", "ws"])
def test_attention_backward_rejects_null_and_unaligned(name):
    assert attention_backward(heads(), **{name: None}) == B.ERR_NULL
    assert attention_backward(heads(), **{name: FAKE + 2}) == B.ERR_ALIGN
    assert attention_backward(None) == B.ERR_NULL and attention_backward(heads(), dt=B.F32) == B.ERR_UNSUPPORTED
    for other in ("s", "ds", "di"):
        assert attention_backward(heads(), **{other: FAKE + 8}) == B.ERR_ALIGN


def test_workspaces():
    h = heads(n_seqs=1, n_tokens=8192, n_heads=64)
    assert 0 <= B.rwkvq_linear_attention_workspace_size(h) < 1 << 30
    assert 0 < B.rwkvq_linear_attention_backward_workspace_size(h) < 1 << 31
    assert 0 < B.rwkvq_layer_norm_backward_workspace_size(8192, 1, 4096) < 1 << 28
    assert B.rwkvq_layer_norm_backward_workspace_size(0, 1, 4096) == 0 and B.rwkvq_layer_norm_backward_workspace_size(1, 1, 0) == 0
    call = B.rwkvq_linear_attention_workspace_size(h)
    assert attention(h, ws=None) == B.ERR_NULL if call else True


def test_heads_struct_layout_matches_header():
    assert ctypes.sizeof(B.rwkvq_heads) == 6 * 4 + 2 * 8 + 4 * 8 and B.rwkvq_heads.offsets.offset == 24
