"""Projections whose every sum is exact, in any order, so that results are compared bit for bit.

X and W hold small integers (X mostly zeros), the scales of e4m3 are powers of two, and Y is an integer that bf16
holds.  Whatever is left out (a k slice, the last k of a row, an adapter, some bits of X A_a) changes Y by a whole
number, however long k is; a bound on the rounding of a sum grows with k and would hide it."""
import torch

from layer_input_ref import E4M3

BF = torch.bfloat16


def exact_case(seed, T, k, n, N, r, fp8=False, wide=False, device="cuda"):
    """Inputs of one projection as keyword arguments.  A row of X has up to 40 nonzeros: some among the last 16 k,
    some next to multiples of 32, the others one in each twentieth of k.  ``wide``: the entries of X A_a need up to 14 bits and cancel
    in pairs of ranks to small ones."""
    g = torch.Generator().manual_seed(seed)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=g)

    edge = (32 * ints(0, (k - 1) // 32, T, 12) - ints(0, 1, T, 12)).clamp(0, k - 1)
    every = (k * (torch.arange(20) + torch.rand(T, 20, generator=g)) / 20).long().clamp(0, k - 1)   # each twentieth of k
    at = torch.cat([every, edge, k - 1 - ints(0, min(15, k - 1), T, 7), torch.full((T, 1), k - 1)], 1)
    X = torch.zeros(T, k).scatter_(1, at, (2 * ints(0, 1, T, 40) - 1).float())
    X[:, k - 1] = 1.0
    W = 2.0 * ints(0, 1, k, n) - 1
    c = {}
    if fp8:
        c["X"], c["W"] = X.to(E4M3), W.to(E4M3)
        c["x_scale"], c["w_scale"] = 2.0 ** (ints(0, 4, T) - 2), 2.0 ** (ints(0, 4, n) - 2)
    else:
        c["X"], c["W"] = X.to(BF), W.to(BF)
    small = ints(-1, 1, k, N, r).float()
    small[k - 1] = 1.0
    B = torch.zeros(N, r, n)
    col = torch.arange(n)
    for a in range(N):
        p = (col + a) % (r // 2) * 2      # each pair of ranks in turn
        if wide:
            B[a, p, col], B[a, p + 1, col] = 1.0, -1.0
        else:
            B[a, p + (col // r) % 2, col] = 1.0
    A = small
    if wide:
        A = (ints(129, 254, k, N, r) * (2 * ints(0, 1, k, N, r) - 1)).float()
        A[:, :, 1::2] = A[:, :, 0::2] + small[:, :, 1::2]   # |A| <= 255: whole numbers of bf16
    c["A_stack"], c["B"] = A.reshape(k, N * r).to(BF), B.to(BF)
    c["agent"] = ints(-1, N - 1, T).to(torch.int32)
    c["agent"][T // 2] = N - 1
    if fp8:   # the adapters' part is scaled by x_scale alone: B takes w_scale's powers of two
        c["B"] = (B * c["w_scale"]).to(BF)
    return {key: v.to(device) for key, v in c.items()}


def exact_y(c, bf16_rows=False, keep=None, adapters=True):
    """Y in float64.  The other arguments leave something out: bits of X A_a, all k but those of the mask ``keep``,
    the adapters."""
    X, W = c["X"].double(), c["W"].double()
    if keep is not None:
        X = X * keep.to(X.device)
    Y = X @ W
    if "x_scale" in c:
        X = X * c["x_scale"].double()[:, None]
        Y = Y * c["x_scale"].double()[:, None] * c["w_scale"].double()
    r = c["B"].shape[1]
    for a in range(c["B"].shape[0] if adapters else 0):
        i = (c["agent"] == a).nonzero().flatten()
        H = X[i] @ c["A_stack"][:, a * r:(a + 1) * r].double()
        Y[i] += (H.to(BF).double() if bf16_rows else H) @ c["B"][a].double()
    return Y
