"""More rows than one grid holds (a grid has fewer than 2^32 threads): the rows of a short input, again and again."""
import pytest
import torch

import paper_2609_34054_amd as prc
from layer_input_exact import exact_case, exact_y
from layer_input_ref import Draws, call as project, check_norm, check_norm_fp8

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
N = 4096   # different rows


def again(t, T):
    """T rows: those of t in turn."""
    out = torch.empty((T,) + t.shape[1:], dtype=t.dtype, device=t.device)
    whole = T // N * N
    out[:whole].view((T // N,) + t.shape).copy_(t.expand((T // N,) + t.shape))
    out[whole:] = t[:T - whole]
    return out


def same(got, t):
    """Whether got holds the rows of t in turn, bit for bit (looked at in pieces)."""
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]
    got, t = got.view(kind), t.view(kind)
    piece = max(1, (1 << 28) // t.numel()) * N
    for i in range(0, len(got), piece):
        p = got[i:i + piece]
        whole = len(p) // N * N
        if not (p[:whole].view((whole // N,) + t.shape) == t).all() or not torch.equal(p[whole:], t[:len(p) - whole]):
            return False
    return True


@pytest.mark.parametrize("T,d,fp8", [((1 << 26) + 3, 8, False), ((1 << 26) + 3, 16, True), ((1 << 24) + 3, 1032, False)])
def test_norm_of_more_rows_than_a_grid_holds(T, d, fp8):
    print(f"norm {T} {d} fp8={fp8}", flush=True)
    rnd = Draws(d)
    x, res, w = rnd.bf16(N, d), rnd.bf16(N, d, std=3.0), (1 + rnd(d, std=0.1)).to(BF)
    call = prc.add_rms_norm_fp8 if fp8 else prc.add_rms_norm
    want = call(x, w, res)
    if fp8:
        check_norm_fp8(want[0], want[1], x, w, res, 1e-5, want[2])
    else:
        check_norm(want[0], x, w, res, 1e-5, want[1])
    long_x, long_res = again(x, T), again(res, T)
    got = call(long_x, w, long_res, residual_out=long_res)
    for g, v in zip(got, want):
        assert same(g, v)
    del long_x, long_res, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,k,n,r,fp8", [((1 << 29) + 77, 8, 8, 8, False), ((1 << 29) + 77, 16, 16, 8, True),
                                         ((1 << 20) + 77, 8, (1 << 15) + 64, 16, False)])
def test_projection_of_more_rows_than_a_grid_holds(T, k, n, r, fp8):
    print(f"project {T} {k} {n} r{r} fp8={fp8}", flush=True)
    c = exact_case(T + k, N, k, n, 3, r, fp8)
    want = exact_y(c).to(BF)
    assert torch.equal(project(prc, c), want)
    long = dict(c, X=again(c["X"].view(torch.int8 if fp8 else torch.int16), T).view(c["X"].dtype), agent=again(c["agent"], T))
    if fp8:
        long["x_scale"] = again(c["x_scale"], T)
    assert same(project(prc, long), want)
    del long
    torch.cuda.empty_cache()


def test_workspace_of_more_rows_than_a_grid_holds():
    """No larger than the parts it goes in need."""
    size = prc.adapted_projection_workspace_size
    assert size((1 << 29) + 77, 8, 8, 3, 8) <= (1 << 28) * 8 * 4
    assert size((1 << 31) - 1, 64, 8, 3, 64) <= (1 << 28) * 64 * 4
