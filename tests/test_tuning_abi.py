"""CPU-side checks of the entry points of dropout, embeddings and adapters: refusals before anything is launched, workspace sizes, the host
structs' layout."""
import ctypes

import pytest

from paper_2505_03803_amd import binding as B

FAKE = 0x10000          # a non-null, 16-byte aligned address that is never dereferenced
OTHER = 0x20000


def dropout(**kw):
    a = dict(x=FAKE, dt=B.BF16, M=4, n=64, xs=0, seed=FAKE, p=0.1, base=None, bs=0, y=OTHER, ys=0)
    a.update(kw)
    return B.lib().rwkvq_dropout(a["x"], a["dt"], a["M"], a["n"], a["xs"], a["seed"], a["p"], a["base"], a["bs"], a["y"], a["ys"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), B.ERR_NULL), (dict(y=None), B.ERR_NULL), (dict(seed=None), B.ERR_NULL), (dict(dt=3), B.ERR_UNSUPPORTED),
    (dict(p=-0.1), B.ERR_UNSUPPORTED), (dict(p=1.1), B.ERR_UNSUPPORTED), (dict(p=float("nan")), B.ERR_UNSUPPORTED),
    (dict(M=0), B.ERR_SHAPE), (dict(n=0), B.ERR_SHAPE), (dict(n=(1 << 24) + 1), B.ERR_SHAPE), (dict(xs=63), B.ERR_SHAPE),
    (dict(ys=-1), B.ERR_SHAPE), (dict(bs=8), B.ERR_SHAPE), (dict(xs=1 << 40), B.ERR_SHAPE),
    (dict(y=FAKE, ys=72), B.ERR_SHAPE), (dict(base=OTHER, ys=72), B.ERR_SHAPE),
    (dict(x=FAKE + 2), B.ERR_ALIGN), (dict(y=OTHER + 8), B.ERR_ALIGN), (dict(base=FAKE + 4), B.ERR_ALIGN), (dict(seed=FAKE + 4), B.ERR_ALIGN),
    (dict(y=FAKE + 8, xs=72), B.ERR_ALIGN),
])
def test_dropout_rejects(kw, status):
    assert dropout(**kw) == status


def embedding(**kw):
    a = dict(tokens=FAKE, T=5, table=FAKE, tdt=B.F16, vocab=100, d=64, scale=1.0, out=FAKE, odt=B.F16, os=0)
    a.update(kw)
    return B.lib().rwkvq_embedding(a["tokens"], a["T"], a["table"], a["tdt"], a["vocab"], a["d"], a["scale"], a["out"], a["odt"], a["os"], None)


def embedding_backward(**kw):
    a = dict(tokens=FAKE, T=5, dout=FAKE, dt=B.F16, ds=0, vocab=100, d=64, scale=1.0, dtable=FAKE, acc=0, ws=FAKE)
    a.update(kw)
    return B.lib().rwkvq_embedding_backward(a["tokens"], a["T"], a["dout"], a["dt"], a["ds"], a["vocab"], a["d"], a["scale"], a["dtable"], a["acc"],
                                            a["ws"], None)


COMMON = [(dict(tokens=None), B.ERR_NULL), (dict(T=0), B.ERR_SHAPE), (dict(vocab=0), B.ERR_SHAPE), (dict(d=0), B.ERR_SHAPE),
          (dict(d=(1 << 24) + 1), B.ERR_SHAPE), (dict(vocab=1 << 30, d=1 << 20), B.ERR_SHAPE), (dict(scale=float("inf")), B.ERR_UNSUPPORTED),
          (dict(scale=float("nan")), B.ERR_UNSUPPORTED), (dict(scale=1e60), B.ERR_UNSUPPORTED), (dict(tokens=FAKE + 2), B.ERR_ALIGN)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(table=None), B.ERR_NULL), (dict(out=None), B.ERR_NULL), (dict(tdt=5), B.ERR_UNSUPPORTED), (dict(odt=-1), B.ERR_UNSUPPORTED),
    (dict(os=63), B.ERR_SHAPE), (dict(os=1 << 40), B.ERR_SHAPE), (dict(table=FAKE + 8), B.ERR_ALIGN), (dict(out=FAKE + 2), B.ERR_ALIGN)])
def test_embedding_rejects(kw, status):
    assert embedding(**kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(dout=None), B.ERR_NULL), (dict(dtable=None), B.ERR_NULL), (dict(ws=None), B.ERR_NULL), (dict(dt=3), B.ERR_UNSUPPORTED),
    (dict(ds=60), B.ERR_SHAPE), (dict(T=(1 << 22) + 1), B.ERR_SHAPE), (dict(T=1 << 22, d=1 << 18, vocab=8), B.ERR_SHAPE),
    (dict(dout=FAKE + 8), B.ERR_ALIGN), (dict(dtable=FAKE + 4), B.ERR_ALIGN), (dict(ws=FAKE + 8), B.ERR_ALIGN)])
def test_embedding_backward_rejects(kw, status):
    assert embedding_backward(**kw) == status


ROWS = dict(n_seqs=2, n_tokens=10, n_adapters=3, rank=16)
MAT = dict(a=FAKE, b=FAKE, x=FAKE, base=None, y=OTHER, h=None, N=64, K=128, x_stride=0, base_stride=0, y_stride=0)
GRAD = dict(a=FAKE, b=FAKE, x=FAKE, h=FAKE, dy=FAKE, base=None, dx=OTHER, da=FAKE, db=FAKE, N=64, K=128, x_stride=0, dy_stride=0, base_stride=0, dx_stride=0)


def rows(**kw):
    return B.AdapterRows(**{**ROWS, **kw})


def forward(r=None, n=1, dt=B.F16, y_dt=B.BF16, **kw):
    mats = (B.rwkvq_adapter * 65)(*[B.rwkvq_adapter(**{**MAT, **kw})] * 65)
    r = r or rows()
    return B.lib().rwkvq_adapters(r.ref, ctypes.addressof(mats), n, dt, y_dt, None)


def gradient(r=None, n=1, dt=B.BF16, ws=FAKE, **kw):
    mats = (B.rwkvq_adapter_grad * 65)(*[B.rwkvq_adapter_grad(**{**GRAD, **kw})] * 65)
    r = r or rows()
    status = B.lib().rwkvq_adapters_backward(r.ref, ctypes.addressof(mats), n, dt, ws, None)
    return status, B.lib().rwkvq_adapters_backward_workspace_size(r.ref, ctypes.addressof(mats), n)


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=0), B.ERR_SHAPE), (dict(n_tokens=0), B.ERR_SHAPE), (dict(n_adapters=0), B.ERR_SHAPE), (dict(n_adapters=65536), B.ERR_SHAPE),
    (dict(rank=0), B.ERR_SHAPE), (dict(rank=12), B.ERR_UNSUPPORTED), (dict(rank=136), B.ERR_UNSUPPORTED), (dict(n_tokens=11), B.ERR_SHAPE),
    (dict(n_tokens=11, offsets=FAKE + 2), B.ERR_ALIGN), (dict(adapters=FAKE + 1), B.ERR_ALIGN), (dict(scales=FAKE + 2), B.ERR_ALIGN),
    (dict(seed=FAKE + 4, p=0.1), B.ERR_ALIGN), (dict(seed=FAKE, p=-0.5), B.ERR_UNSUPPORTED), (dict(seed=FAKE, p=1.5), B.ERR_UNSUPPORTED),
    (dict(n_seqs=1 << 22, n_tokens=1 << 22), B.ERR_SHAPE),
])
def test_adapter_rows_rejected(kw, status):
    assert forward(rows(**kw)) == status
    assert gradient(rows(**kw)) == (status, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(a=None), B.ERR_NULL), (dict(b=None), B.ERR_NULL), (dict(x=None), B.ERR_NULL), (dict(N=0), B.ERR_SHAPE), (dict(K=-8), B.ERR_SHAPE),
    (dict(N=60), B.ERR_ALIGN), (dict(K=100), B.ERR_ALIGN), (dict(K=(1 << 24) + 8), B.ERR_SHAPE), (dict(x_stride=120), B.ERR_SHAPE),
    (dict(x_stride=132), B.ERR_ALIGN), (dict(x_stride=1 << 40), B.ERR_SHAPE), (dict(n=0), B.ERR_SHAPE), (dict(n=65), B.ERR_SHAPE),
    (dict(a=FAKE + 8), B.ERR_ALIGN), (dict(b=FAKE + 2), B.ERR_ALIGN), (dict(x=FAKE + 4), B.ERR_ALIGN), (dict(h=FAKE + 8), B.ERR_ALIGN),
    (dict(base=FAKE + 8), B.ERR_ALIGN),
])
def test_adapter_matrices_rejected(kw, status):
    assert forward(**kw) == status and gradient(**kw)[0] == status


@pytest.mark.parametrize("kw,status", [
    (dict(y=None), B.ERR_NULL), (dict(y=FAKE), B.ERR_SHAPE), (dict(base=OTHER, y_stride=72), B.ERR_SHAPE), (dict(y_stride=56), B.ERR_SHAPE),
    (dict(y_stride=68), B.ERR_ALIGN), (dict(base_stride=65), B.ERR_ALIGN), (dict(y=OTHER + 8), B.ERR_ALIGN), (dict(dt=B.F32), B.ERR_UNSUPPORTED),
    (dict(y_dt=3), B.ERR_UNSUPPORTED)])
def test_adapters_reject(kw, status):
    assert forward(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(h=None), B.ERR_NULL), (dict(dy=None), B.ERR_NULL), (dict(da=None), B.ERR_NULL), (dict(db=None), B.ERR_NULL), (dict(ws=None), B.ERR_NULL),
    (dict(dx=FAKE), B.ERR_SHAPE), (dict(base=OTHER, dx_stride=136), B.ERR_SHAPE), (dict(dy_stride=56), B.ERR_SHAPE), (dict(dy_stride=68), B.ERR_ALIGN),
    (dict(dx_stride=120), B.ERR_SHAPE), (dict(dx=OTHER + 8), B.ERR_ALIGN), (dict(da=FAKE + 4), B.ERR_ALIGN), (dict(db=FAKE + 8), B.ERR_ALIGN),
    (dict(dy=FAKE + 2), B.ERR_ALIGN), (dict(ws=FAKE + 8), B.ERR_ALIGN), (dict(dt=B.F32), B.ERR_UNSUPPORTED)])
def test_adapters_backward_reject(kw, status):
    assert gradient(**kw)[0] == status


def test_missing_structs():
    L, r = B.lib(), rows()
    assert L.rwkvq_adapters(None, FAKE, 1, B.F16, B.F16, None) == B.ERR_NULL and L.rwkvq_adapters(r.ref, None, 1, B.F16, B.F16, None) == B.ERR_NULL
    assert L.rwkvq_adapters_backward(None, FAKE, 1, B.F16, FAKE, None) == B.ERR_NULL
    assert L.rwkvq_adapters_backward_workspace_size(None, None, 1) == 0


def test_workspaces():
    assert B.rwkvq_embedding_backward_workspace_size(8192, 4096) > 0 and B.rwkvq_embedding_backward_workspace_size(1, 1) > 0
    assert B.rwkvq_embedding_backward_workspace_size(0, 8) == 0 and B.rwkvq_embedding_backward_workspace_size((1 << 22) + 1, 8) == 0
    assert gradient(ws=None)[1] > 0


def test_struct_layouts_match_header():
    assert ctypes.sizeof(B.rwkvq_adapter_rows) == 4 * 4 + 4 * 8 + 8 and B.rwkvq_adapter_rows.offsets.offset == 16
    assert ctypes.sizeof(B.rwkvq_adapter) == 6 * 8 + 2 * 4 + 3 * 8 and B.rwkvq_adapter.N.offset == 48
    assert ctypes.sizeof(B.rwkvq_adapter_grad) == 9 * 8 + 2 * 4 + 4 * 8 and B.rwkvq_adapter_grad.N.offset == 72
