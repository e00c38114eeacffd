"""What the layer-input operators refuse, on the host before any HIP call."""
import pytest
import torch

import paper_2609_34054_amd as prc
from layer_input_ref import E4M3, project_case

OK, EINVAL, ESHAPE, EALIGN, EUNSUP, EWS, EDEVICE = 0, 1, 2, 3, 4, 5, 7
GB = 1 << 30
X, W, A, B, AG, Y, WS, XS, SC = (k * 8 * GB for k in range(1, 10))   # never dereferenced on the host


def _proj(T=64, k=256, ldx=None, n=512, N=3, r=16, ldy=None, X=X, W=W, A=A, B=B, ag=AG, Y=Y, ws=WS, wb=1 << 32):
    return prc.lib().adapted_projection(X, T, k, k if ldx is None else ldx, W, n, A, B, N, r, ag, Y,
                                        n if ldy is None else ldy, ws, wb, None)


def _proj8(T=64, k=256, ldx=None, n=512, N=3, r=16, ldy=None, X=X, xs=XS, W=W, sc=SC, Y=Y):
    return prc.lib().adapted_projection_fp8(X, xs, T, k, k if ldx is None else ldx, W, sc, n, A, B, N, r, AG, Y,
                                            n if ldy is None else ldy, WS, 1 << 32, None)


def _norm(T=8, d=256, ldx=256, res=W, ldr=256, w=A, eps=1e-5, out=B, ldo=256, y=Y, ldy=256, x=X):
    return prc.lib().add_rms_norm(x, T, d, ldx, res, ldr, w, eps, out, ldo, y, ldy, None)


def _norm8(T=8, d=256, ldx=256, res=W, y=Y, ldy=256, ys=XS, out=B):
    return prc.lib().add_rms_norm_fp8(X, T, d, ldx, res, 256, A, 1e-5, out, 256, y, ldy, ys, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(T=1 << 31), EINVAL), (dict(k=0), EUNSUP), (dict(k=260), EUNSUP), (dict(n=0), EUNSUP),
    (dict(n=12), EUNSUP), (dict(N=-1), EINVAL), (dict(r=12), EUNSUP), (dict(r=128), EUNSUP), (dict(r=0), EUNSUP),
    (dict(ldx=248), ESHAPE), (dict(ldy=504), ESHAPE), (dict(ldx=260), EALIGN), (dict(ldy=516), EALIGN),
    (dict(ldx=1 << 22), EUNSUP), (dict(ldy=1 << 22), EUNSUP), (dict(k=1 << 15, n=1 << 15), EUNSUP),
    (dict(k=1 << 14, N=1 << 13, r=16), EUNSUP),
    (dict(T=(1 << 31) - 1, k=8, n=1 << 12), EUNSUP), (dict(k=8, n=1 << 22), EUNSUP), (dict(k=1 << 22, n=8), EUNSUP), (dict(X=None), EINVAL), (dict(W=None), EINVAL), (dict(A=None), EINVAL),
    (dict(B=None), EINVAL), (dict(ag=None), EINVAL), (dict(Y=None), EINVAL), (dict(X=X + 8), EALIGN),
    (dict(W=W + 2), EALIGN), (dict(B=B + 8), EALIGN), (dict(Y=Y + 8), EALIGN), (dict(ag=AG + 2), EALIGN),
    (dict(ws=None), EWS), (dict(wb=16), EWS), (dict(ws=WS + 8), EALIGN), (dict(Y=X), EINVAL), (dict(Y=X + 16384), EINVAL),
    (dict(Y=W), EINVAL), (dict(Y=A), EINVAL), (dict(Y=B), EINVAL), (dict(Y=AG), EINVAL), (dict(Y=WS), EINVAL),
    (dict(ws=X), EINVAL), (dict(Y=X - 64 * 512 * 2 + 16), EINVAL),
])
def test_projection_rejects(kw, code):
    assert _proj(**kw) == code
    assert prc.lib().prc_last_error().decode()


@pytest.mark.parametrize("kw,code", [
    (dict(k=264), EUNSUP), (dict(n=520), EUNSUP), (dict(ldx=264), EALIGN), (dict(xs=None), EINVAL), (dict(sc=None), EINVAL),
    (dict(xs=XS + 2), EALIGN), (dict(Y=XS), EINVAL), (dict(Y=SC), EINVAL),
])
def test_8_bit_projection_rejects(kw, code):
    assert _proj8(**kw) == code
    assert prc.lib().prc_last_error().decode()


@pytest.mark.parametrize("kw", [dict(ldx=1 << 36), dict(ldr=1 << 36), dict(ldo=1 << 36), dict(ldy=1 << 36)])
def test_norm_rejects_rows_beyond_64_bit_offsets(kw):
    assert _norm(T=(1 << 31) - 1, **kw) == EUNSUP
    assert "too many" in prc.lib().prc_last_error().decode()


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(T=1 << 31), EINVAL), (dict(d=0), EUNSUP), (dict(d=252), EUNSUP), (dict(d=65544), EUNSUP),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(ldx=248), ESHAPE),
    (dict(ldr=248), ESHAPE), (dict(ldo=248), ESHAPE), (dict(ldy=248), ESHAPE), (dict(ldx=260), EALIGN),
    (dict(ldy=260), EALIGN), (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(y=None), EINVAL), (dict(x=X + 8), EALIGN),
    (dict(res=W + 8), EALIGN), (dict(out=B + 8), EALIGN), (dict(y=Y + 8), EALIGN), (dict(y=X + 16), EINVAL),
    (dict(y=X, ldy=264), EINVAL), (dict(out=W + 512), EINVAL), (dict(out=A), EINVAL), (dict(y=A), EINVAL),
    (dict(y=B), EINVAL), (dict(y=W, out=W), EINVAL),
])
def test_norm_rejects(kw, code):
    assert _norm(**kw) == code
    assert prc.lib().prc_last_error().decode()


@pytest.mark.parametrize("kw,code", [
    (dict(d=248), EUNSUP), (dict(ldy=264), EALIGN), (dict(ys=None), EINVAL), (dict(ys=XS + 2), EALIGN), (dict(y=X), EINVAL),
    (dict(y=W), EINVAL), (dict(ys=X), EINVAL), (dict(ys=Y), EINVAL), (dict(out=X, ldx=264), EINVAL),
])
def test_8_bit_norm_rejects(kw, code):
    assert _norm8(**kw) == code
    assert prc.lib().prc_last_error().decode()


def test_valid_calls_pass_every_check():
    """They end at the device check, which a host without a GPU fails; with no rows they end before."""
    if not torch.cuda.is_available():
        assert {_proj(), _proj8(), _norm(), _norm8(), _norm(y=X, out=W), _norm(y=W, out=X), _norm(res=None, out=None),
                _proj(N=0, A=None, B=None, ag=None, r=0)} == {EDEVICE}
        assert "device" in prc.lib().prc_last_error().decode()
    assert {_proj(T=0, X=None, W=None), _proj8(T=0, X=None), _norm(T=0, x=None), _norm8(T=0, y=None)} == {OK}


def test_workspace_query():
    size = prc.adapted_projection_workspace_size
    assert size(0, 256, 256, 3, 16) == 0 and size(-1, 256, 256, 3, 16) == 0 and size(64, 256, 256, 3, 12) == 0
    assert size(1 << 31, 256, 256, 3, 16) == 0 and size(64, -8, 256, 3, 16) == 0
    for T in (1, 3, 64, 200, 1000, 4096, 100000):
        for N in (1, 8, 64):
            need = size(T, 4096, 4096, N, 16)
            assert T * 16 * 2 <= need <= (64 << 20) + T * 64
    if not torch.cuda.is_available():
        assert _proj(wb=size(64, 256, 512, 3, 16)) == EDEVICE


# ------------------------------------------------------------ the binding
def _c(**kw):
    c = project_case(1, 6, 64, 32, 3, 8, device="cpu")
    c.update(kw)
    return c


def _call(c):
    return prc.adapted_projection(c["X"], c["W"], c["A_stack"], c["B"], c["agent"], **{k: c[k] for k in ("Y", "workspace") if k in c})


BAD = [
    (lambda c: dict(X=c["X"].float()), TypeError), (lambda c: dict(W=c["W"].half()), TypeError),
    (lambda c: dict(X=c["X"][0]), ValueError), (lambda c: dict(X=c["X"].t().contiguous().t()), ValueError),
    (lambda c: dict(W=c["W"][:, ::2]), ValueError), (lambda c: dict(W=c["W"][:32]), ValueError),
    (lambda c: dict(A_stack=c["A_stack"][:, :16]), ValueError), (lambda c: dict(B=c["B"][:, :, :24]), ValueError),
    (lambda c: dict(B=c["B"][0]), ValueError), (lambda c: dict(agent=c["agent"][:5]), ValueError),
    (lambda c: dict(agent=c["agent"].long()), TypeError), (lambda c: dict(agent=None), ValueError),
    (lambda c: dict(A_stack=None), ValueError), (lambda c: dict(Y=torch.empty((6, 24), dtype=torch.bfloat16)), ValueError),
    (lambda c: dict(Y=torch.empty((6, 32))), TypeError),
    (lambda c: dict(workspace=torch.empty(64, dtype=torch.uint8)[::2]), ValueError),
    (lambda c: {}, ValueError),   # not on a GPU
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_binding_rejects(i):
    make, err = BAD[i]
    c = _c()
    with pytest.raises(err):
        _call(dict(c, **make(c)))


def test_8_bit_binding_rejects():
    c = project_case(1, 6, 64, 32, 3, 8, fp8=True, device="cpu")
    ok = (c["X"], c["x_scale"], c["W"], c["w_scale"], c["A_stack"], c["B"], c["agent"])
    for i, bad, err in ((0, c["X"].float(), TypeError), (1, c["x_scale"][:5], ValueError), (1, c["x_scale"].double(), TypeError),
                        (2, c["W"].to(torch.bfloat16), TypeError), (3, c["w_scale"][:16], ValueError), (0, c["X"], ValueError)):
        args = list(ok)
        args[i] = bad
        with pytest.raises(err):
            prc.adapted_projection_fp8(*args)


def test_norm_binding_rejects():
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    for args, kw, err in (((x.float(), w), {}, TypeError), ((x, w[:32]), {}, ValueError), ((x, w.float()), {}, TypeError),
                          ((x[0], w), {}, ValueError), ((x, w, x[:3]), {}, ValueError), ((x, w, x.half()), {}, TypeError),
                          ((x, w), dict(y=x.to(E4M3)), TypeError), ((x, w), dict(residual_out=x[:2]), ValueError),
                          ((x.t(), w), {}, ValueError), ((x, w), {}, ValueError)):
        with pytest.raises(err):
            prc.add_rms_norm(*args, **kw)
    for kw, err in ((dict(y=x), TypeError), (dict(y_scale=torch.zeros(4).double()), TypeError),
                    (dict(y_scale=torch.zeros(3)), ValueError), ({}, ValueError)):
        with pytest.raises(err):
            prc.add_rms_norm_fp8(x, w, **kw)
