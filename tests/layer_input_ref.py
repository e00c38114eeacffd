"""Plain 64-bit forms of the layer-input operators, with elementwise error bounds.

A bound counts roundings: half a step of a type relative to the value (bf16
2^-8, e4m3 2^-4, of its subnormals 2^-10 absolute), and for a sum of n terms in
fp32, in any order, n * 2^-23 of the sum of the terms' sizes (2^-24 a rounding,
doubled for matrix instructions that may cut instead of round).

The e4m3 matrix instructions sum eight products at a time, each cut (towards
zero) to a multiple of 2^-13 of the largest one's power of two before they are
added in fp32 (seen on gfx950 by adding a product of 2^e to one of 2^16: 2^3
arrives, 2^2 does not, within the same eight k; in another eight both do).  So a
group of eight loses at most 7 * 2^-13 of its largest product, which is no more
than 7 * 2^-13 of the sum of its products' sizes."""
import torch

U8, UF = 2.0 ** -8, 2.0 ** -23
U_E4M3 = 7 * 2.0 ** -13
E4M3 = torch.float8_e4m3fn


def norm_ref(x, weight, residual, eps):
    """(y, s) in float64 and the relative error y may have before its rounding."""
    s = x.double() + (0.0 if residual is None else residual.double())
    ms = s.square().mean(1, keepdim=True)
    y = s / torch.sqrt(ms + eps) * weight.double()
    # s: 2^-24; its square's sum: at most 200 roundings deep (64 a thread, the lanes and waves, the mean); root,
    # reciprocal and two products: 5.
    return y, s, 210 * 2.0 ** -24


def check_norm(got, x, weight, residual, eps, out=None):
    y, s, rel = norm_ref(x, weight, residual, eps)
    if out is not None:
        assert torch.all((out.double() - s).abs() <= s.abs() * (U8 + 2.0 ** -23)), "residual_out"
    err = (got.double() - y).abs()
    tol = y.abs() * (U8 + 2 * rel) + 2.0 ** -133
    assert torch.all(err <= tol), float((err / tol).max())


def check_norm_fp8(q, scale, x, weight, residual, eps, out=None):
    y, s, rel = norm_ref(x, weight, residual, eps)
    if out is not None:
        assert torch.all((out.double() - s).abs() <= s.abs() * (U8 + 2.0 ** -23)), "residual_out"
    want = y.abs().amax(1).clamp_min(2.0 ** -100) / 448
    assert torch.all((scale.double() - want).abs() <= want * (rel + 2.0 ** -23)), "scale"
    sc = scale.double()[:, None]
    err = (q.double() * sc - y).abs()
    # Half a step, and what y and the quotient were off by before it.
    tol = (y.abs() * 2.0 ** -4 + sc * 2.0 ** -10) * (1 + 4 * rel) + y.abs() * 4 * rel
    assert torch.all(err <= tol), float((err / tol).max())


def project_ref(X, W, A, B, agent, x_scale=None, w_scale=None):
    """Y in float64 and its elementwise bound (a rounding of Y among it)."""
    X, W = X.double(), W.double()
    k = X.shape[1]
    sc = 1.0
    if x_scale is not None:
        sc = x_scale.double()[:, None] * w_scale.double()[None, :]
    Y, bound = X @ W * sc, (X.abs() @ W.abs()) * sc * ((k + 4) * UF + (0.0 if x_scale is None else U_E4M3))
    for a in range(0 if B is None else B.shape[0]):
        i = (agent == a).nonzero().flatten()
        if not len(i):
            continue
        r = B.shape[1]
        Aa, Ba = A[:, a * r:(a + 1) * r].double(), B[a].double()
        Xa = X[i] if x_scale is None else X[i] * x_scale.double()[i, None]
        H, Habs = Xa @ Aa, Xa.abs() @ Aa.abs()
        dH = Habs * ((k + 2) * UF) + H.abs() * U8 * (1 + U8)   # sums, the rounding to bf16
        Y[i] += H @ Ba
        bound[i] += dH @ Ba.abs() * (1 + U8) + (H.abs() @ Ba.abs()) * ((r + 4) * UF)
    return Y, (bound + Y.abs() * U8) * (1 + U8) + 2.0 ** -133


def check_project(got, ref, bound):
    err = (got.double() - ref).abs()
    assert torch.isfinite(got.float()).all()
    assert torch.all(err <= bound), float((err / bound).max())


def quantised(x, dim):
    """x in e4m3 with fp32 scales over `dim`."""
    scale = x.abs().amax(dim).clamp_min(2.0 ** -100) / 448
    return (x / scale.unsqueeze(dim)).clamp(-448, 448).to(E4M3), scale


class Draws:
    def __init__(self, seed, device="cuda"):
        self.g, self.device = torch.Generator().manual_seed(seed), device

    def __call__(self, *shape, std=1.0):
        return (torch.randn(shape, generator=self.g) * std).to(self.device)

    def bf16(self, *shape, std=1.0):
        return self(*shape, std=std).to(torch.bfloat16)

    def ints(self, lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=self.g).to(torch.int32).to(self.device)


def project_case(seed, T, k, n, N, r, order="mixed", fp8=False, device="cuda"):
    """Inputs of one projection as keyword arguments; ``order``: "mixed", "runs",
    "one" (a single agent), "none" (base rows alone), "some" (base rows among
    mixed ones, some of them by an entry past the last agent)."""
    rnd = Draws(seed, device)
    X, W = rnd(T, k), rnd(k, n, std=k ** -0.5)
    c = {}
    if fp8:
        c["X"], c["x_scale"] = quantised(X, 1) if T else (X.to(E4M3), X.new_zeros(0))
        c["W"], c["w_scale"] = quantised(W, 0)
    else:
        c["X"], c["W"] = X.to(torch.bfloat16), W.to(torch.bfloat16)
    c["A_stack"] = rnd.bf16(k, N * r, std=k ** -0.5) if N else None
    c["B"] = rnd.bf16(N, r, n, std=0.14) if N else None
    if not N:
        c["agent"] = None
    elif order == "mixed":
        c["agent"] = rnd.ints(0, N, T)
    elif order == "some":
        c["agent"] = rnd.ints(-2, N + 2, T)
    elif order == "none":
        c["agent"] = torch.full((T,), -1, dtype=torch.int32, device=device)
    elif order == "one":
        c["agent"] = torch.full((T,), N - 1, dtype=torch.int32, device=device)
    else:
        c["agent"] = (torch.arange(T) * 5 // max(T, 1) % N).to(torch.int32).to(device)
    return c


def ref_of(c):
    return project_ref(c["X"], c["W"], c["A_stack"], c["B"], c["agent"], c.get("x_scale"), c.get("w_scale"))


def call(prc, c, **kw):
    if "x_scale" in c:
        return prc.adapted_projection_fp8(c["X"], c["x_scale"], c["W"], c["w_scale"], c["A_stack"], c["B"], c["agent"], **kw)
    return prc.adapted_projection(c["X"], c["W"], c["A_stack"], c["B"], c["agent"], **kw)
