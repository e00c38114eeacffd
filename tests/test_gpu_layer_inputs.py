"""The layer-input operators (residual RMS norm, projections with per-row
adapters, in bf16 and 8 bits) against their plain 64-bit forms."""
import pytest
import torch

import paper_2609_34054_amd as prc
from layer_input_ref import (E4M3, Draws, call, check_norm, check_norm_fp8, check_project, norm_ref, project_case, ref_of)

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


# ------------------------------------------------------------------- norm
NORM_SHAPES = [(1, 8), (1, 16), (3, 24), (1, 4096), (2, 5120), (7, 256), (5, 8192), (3, 8208), (2, 65536), (1, 32784),
               (64, 4096), (257, 512), (1000, 4096), (1025, 80), (1500, 5120), (2049, 8192), (1100, 8208), (5000, 16)]


def norm_case(T, d, residual, seed=0):
    rnd = Draws(1000 * T + d + seed)
    x, w = rnd.bf16(T, d), (1 + rnd(d, std=0.1)).to(BF)
    return x, w, (rnd(T, d) * 4).to(BF) if residual else None


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("T,d", NORM_SHAPES)
def test_norm(T, d, residual):
    print(f"norm {T} {d} {residual}", flush=True)
    x, w, res = norm_case(T, d, residual)
    y, out = prc.add_rms_norm(x, w, res, eps=1e-5)
    check_norm(y, x, w, res, 1e-5, out)
    if d % 16 == 0:
        q, scale, out8 = prc.add_rms_norm_fp8(x, w, res, eps=1e-5)
        check_norm_fp8(q, scale, x, w, res, 1e-5, out8)
    assert residual or out is None


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("T", [3, 1031])
@pytest.mark.parametrize("d", [504, 512, 520, 1024, 1032, 2048, 2064, 4096, 4112, 16384, 16400, 32768])
def test_norm_widths(T, d, residual):
    """Ends of what a row's threads hold, whole and ragged, with a workgroup's last rows missing."""
    test_norm(T, d, residual)


def test_norm_of_strided_rows_leaves_the_gaps():
    T, d = 37, 264
    x, w, res = norm_case(T, d, True)
    wide = [torch.full((T, d + p), 7.0, dtype=BF, device="cuda") for p in (8, 56, 16, 24)]
    xs, rs, ys, os_ = (t[:, :d] for t in wide)
    xs.copy_(x)
    rs.copy_(res)
    y, out = prc.add_rms_norm(xs, w, rs, y=ys, residual_out=os_)
    check_norm(y, x, w, res, 1e-5, out)
    for t in wide:
        assert torch.all(t[:, d:] == 7.0)
    assert torch.equal(xs, x) and torch.equal(rs, res)


def test_norm_in_place():
    x, w, res = norm_case(33, 512, True)
    want, s = prc.add_rms_norm(x, w, res)
    r2, x2 = res.clone(), x.clone()
    y, out = prc.add_rms_norm(x2, w, r2, y=x2, residual_out=r2)
    assert torch.equal(y, want) and torch.equal(r2, s) and out is r2 and y is x2


def test_norm_writes_a_residual_it_was_not_given():
    x, w, _ = norm_case(5, 64, False)
    out = torch.empty_like(x)
    prc.add_rms_norm(x, w, residual_out=out)
    assert torch.equal(out, x)


def test_norm_of_zero_and_tiny_rows():
    T, d = 4, 256
    x = torch.zeros((T, d), dtype=BF, device="cuda")
    x[1] = 1e-30
    x[2, 3] = 2.0
    w = torch.ones(d, dtype=BF, device="cuda")
    y, _ = prc.add_rms_norm(x, w)
    check_norm(y, x, w, None, 1e-5)
    q, scale, _ = prc.add_rms_norm_fp8(x, w)
    check_norm_fp8(q, scale, x, w, None, 1e-5)
    # 1/448 = 2^-6/7 has no finite binary form: its fp32 value is off by up to half a step, 2^-24.
    assert torch.all(q[0].float() == 0) and abs(float(scale[0]) * 448 * 2.0 ** 100 - 1) <= 2.0 ** -24
    assert float(q[2, 3].float()) == 448.0


def test_norm_keeps_bad_values_in_their_rows():
    T, d = 9, 512
    x, w, res = norm_case(T, d, True)
    good, s = prc.add_rms_norm(x, w, res)
    g8, gs, _ = prc.add_rms_norm_fp8(x, w, res)
    x[4, 17] = float("nan")
    res[6, 300] = float("inf")
    y, out = prc.add_rms_norm(x, w, res)
    q, scale, _ = prc.add_rms_norm_fp8(x, w, res)
    fine = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y[fine], good[fine]) and torch.equal(out[fine], s[fine])
    assert torch.equal(q[fine].float(), g8[fine].float()) and torch.equal(scale[fine], gs[fine])
    assert torch.isnan(y[4].float()).all() and torch.isnan(q[4].float()).all() and torch.isnan(scale[4])
    # An infinite element: its row's root is infinite, so the others vanish and it is infinity times zero.
    assert torch.isnan(y[6, 300].float()) and torch.all(y[6, :300] == 0)
    assert torch.isnan(q[6].float()).all() and torch.isnan(scale[6])


def test_norm_of_no_rows():
    x = torch.empty((0, 64), dtype=BF, device="cuda")
    w = torch.ones(64, dtype=BF, device="cuda")
    assert prc.add_rms_norm(x, w)[0].shape == (0, 64)
    assert prc.add_rms_norm_fp8(x, w, x)[1].shape == (0,)


# ------------------------------------------------------------- projection
ROWS = [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 33, 48, 64, 65, 100, 127, 128, 129, 200, 256, 257, 300, 511, 513, 777, 1025]
SHAPES = [(256, 256), (264, 136), (8, 8), (1032, 72), (40, 520)]
SHAPES8 = [(256, 256), (272, 144), (16, 16), (1040, 80), (48, 528)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", ROWS)
def test_projection_rows(T, fp8):
    for j, order in enumerate(("mixed", "runs", "some")):
        k, n = (SHAPES8 if fp8 else SHAPES)[(T + j) % len(SHAPES)]
        r = (8, 16, 32, 64)[(T + 2 * j) % 4]
        print(f"project {T} {k} {n} r{r} {order} fp8={fp8}", flush=True)
        c = project_case(T + j, T, k, n, 5, r, order, fp8)
        check_project(call(prc, c), *ref_of(c))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n,N,r,order", [
    (1, 4096, 4096, 8, 16, "mixed"), (16, 4096, 4096, 8, 16, "mixed"), (8, 5120, 5120, 6, 64, "mixed"),
    (3, 8192, 1024, 3, 32, "mixed"), (64, 512, 8192, 32, 8, "mixed"), (70, 4112, 4112, 64, 16, "mixed"),
    (512, 4096, 1024, 4, 16, "one"), (1000, 1024, 4096, 8, 8, "runs"), (1, 16, 65536, 2, 64, "mixed"),
    (2048, 2048, 2048, 8, 16, "runs"), (2500, 1040, 2064, 3, 64, "some"), (4097, 512, 4096, 1, 32, "one"),
    (1300, 4096, 4096, 40, 16, "mixed"), (640, 65536, 64, 2, 16, "mixed"), (5000, 64, 64, 6, 64, "runs"),
    (600, 2048, 4096, 300, 8, "mixed"),
])
def test_projection_sizes(T, k, n, N, r, order, fp8):
    print(f"project {T} {k} {n} {N} r{r} {order} fp8={fp8}", flush=True)
    c = project_case(T + k + n, T, k, n, N, r, order, fp8)
    check_project(call(prc, c), *ref_of(c))


# Sizes whose rounds of the CUs favour each of the tile shapes (128 x 64 to 256 x 256), with ends inside tiles.
SHAPES_TILES = [(65, 272, 528), (1000, 1024, 4096), (2500, 1040, 2064), (2040, 272, 5120), (2040, 528, 6144),
                (4090, 272, 4080), (3000, 528, 4096)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("N,r,order", [(3, 64, "some"), (9, 16, "runs"), (1, 32, "one"), (12, 8, "mixed"), (0, 0, "none")])
@pytest.mark.parametrize("T,k,n", SHAPES_TILES)
def test_projection_tile_shapes(T, k, n, N, r, order, fp8):
    print(f"project {T} {k} {n} {N} r{r} {order} fp8={fp8}", flush=True)
    c = project_case(T + k + n + r, T, k, n, N, r, order, fp8)
    check_project(call(prc, c), *ref_of(c))


# A few hundred rows as 64-row slabs: one and several k slices, ends inside a slab, a stage and 16 columns; more
# agents among 64 rows than are taken at once; 128 x 64 tiles where there are too many slabs.
SHAPES_SLABS = [(17, 136, 72), (47, 4112, 272), (64, 64, 4096), (66, 1032, 3080), (191, 2056, 1032), (257, 5128, 520),
                (1000, 1096, 200), (1024, 72, 1048), (300, 3592, 4096), (90, 520, 40000), (1100, 1032, 136), (4090, 520, 64)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("N,r,order", [(200, 64, "mixed"), (9, 32, "some"), (40, 16, "mixed"), (30, 8, "mixed"), (0, 0, "none")])
@pytest.mark.parametrize("T,k,n", SHAPES_SLABS)
def test_projection_slab_shapes(T, k, n, N, r, order, fp8):
    if fp8:
        k, n = (k + 15) // 16 * 16, (n + 15) // 16 * 16
    print(f"project {T} {k} {n} {N} r{r} {order} fp8={fp8}", flush=True)
    c = project_case(T + k + n + r, T, k, n, N, r, order, fp8)
    got = call(prc, c)
    check_project(got, *ref_of(c))
    assert torch.equal(got, call(prc, c))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n", SHAPES_TILES[1:6])
def test_bad_adapters_stay_in_their_rows_of_wide_tiles(T, k, n, fp8):
    for order, r in (("mixed", 16), ("runs", 64)):
        c = project_case(T + r, T, k, n, 4, r, order, fp8)
        want = call(prc, c)
        bad = dict(c, B=c["B"].clone())
        a = int(c["agent"][T // 2])
        bad["B"][a, 5] = float("inf")
        got = call(prc, bad)
        mine = c["agent"] == a
        assert torch.equal(got[~mine], want[~mine]) and (~torch.isfinite(got[mine].float())).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 20, 130, 700])
def test_projection_without_adapters(T, fp8):
    c = project_case(3, T, 512, 272, 0, 0, fp8=fp8)
    check_project(call(prc, c), *ref_of(c))
    d = project_case(3, T, 512, 272, 3, 16, "none", fp8=fp8)
    assert torch.equal(call(prc, d), call(prc, dict(d, A_stack=None, B=None, agent=None)))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 13, 64, 300, 1100])
def test_projection_of_strided_rows_leaves_the_gaps(T, fp8):
    k, n = 272, 528
    c = project_case(T, T, k, n, 4, 16, "some", fp8)
    want = call(prc, c)
    pad = 48
    wide = torch.full((T, k + pad), 3.0, device="cuda").to(c["X"].dtype)
    wide[:, :k] = c["X"]
    Y = torch.full((T, n + 24), 7.0, dtype=BF, device="cuda")
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")   # NaN in every type
    got = call(prc, dict(c, X=wide[:, :k]), Y=Y[:, :n], workspace=ws)
    assert torch.equal(got, want) and torch.all(Y[:, n:] == 7.0)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 3, 40, 129, 600, 1100])
def test_bad_values_stay_in_their_rows(T, fp8):
    """What is infinite or NaN in an adapter, or in a row of X, shows in the rows that use it and in no other."""
    for order in ("mixed", "runs"):
        c = project_case(T + 5, T, 528, 272, 4, 16, order, fp8)
        want = call(prc, c)
        for name in ("A_stack", "B", "X"):
            d = dict(c)
            bad = d[name] = d[name].clone()
            if name == "X":
                mine = torch.zeros(T, dtype=torch.bool, device="cuda")
                mine[T // 2] = True
                bad[T // 2, 100] = float("nan")
            else:
                mine = c["agent"] == int(c["agent"][T // 2])
                a = int(c["agent"][T // 2])
                if name == "A_stack":
                    bad[77, 16 * a + 3] = float("inf")
                else:
                    bad[a, 5] = float("nan")
            got = call(prc, d)
            assert torch.equal(got[~mine], want[~mine]), (order, name)
            assert (~torch.isfinite(got[mine].float())).any(1).all(), (order, name)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 16, 100, 513, 1200])
def test_projection_gives_the_same_bits_again(T, fp8):
    c = project_case(T, T, 2048, 1040, 6, 16, "mixed", fp8)
    want = call(prc, c)
    for _ in range(3):
        assert torch.equal(call(prc, c), want)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [3, 40])
def test_projection_among_very_many_adapters(T, fp8):
    """Rows of A of 32 MB (offsets of a stage's rows past d_in exceed 32 bits): the bits of a call that has only the
    adapters in use."""
    k, n, N, r = 16, 32, 1 << 18, 64
    c = project_case(T, T, k, n, T, r, "mixed", fp8)
    c["agent"] = torch.arange(T, dtype=torch.int32, device="cuda").flip(0)
    where = (torch.arange(T, device="cuda") * (N - 1)) // (T - 1)
    A = torch.full((k, N, r), float("nan"), dtype=BF, device="cuda")
    B = torch.full((N, r, n), float("nan"), dtype=BF, device="cuda")
    A[:, where], B[where] = c["A_stack"].view(k, T, r), c["B"]
    many = dict(c, A_stack=A.view(k, N * r), B=B, agent=where[c["agent"].long()].int())
    want = call(prc, c)
    check_project(want, *ref_of(c))
    assert torch.equal(call(prc, many), want)


def test_projection_of_no_rows():
    c = project_case(1, 0, 64, 48, 2, 8)
    assert call(prc, c).shape == (0, 48)


@pytest.mark.parametrize("T", [1, 24, 300, 1100])
def test_side_stream_and_graphs(T):
    """Work ordered on a stream other than the default; two captured graphs of their own workspaces, replayed in
    turn with eager calls between."""
    cs = [project_case(T + i, T, 512, 528, 4, 16, "mixed", fp8=bool(i)) for i in range(2)]
    nrm = norm_case(T, 512, True)
    want = [call(prc, c) for c in cs]
    wy, ws_ = prc.add_rms_norm(*nrm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [call(prc, c) for c in cs]
    direct = call(prc, cs[0], stream=side)
    side.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.equal(direct, want[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for c in cs:
        Y = torch.zeros_like(want[0])
        size = prc.adapted_projection_workspace_size(T, 512, 528, 4, 16)
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        y, out = torch.zeros_like(nrm[0]), torch.zeros_like(nrm[0])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            prc.add_rms_norm(*nrm, y=y, residual_out=out)
            call(prc, c, Y=Y, workspace=ws)
        graphs.append((g, Y, ws, y, out))
    for rep in range(3):
        for i, (g, Y, ws, y, out) in enumerate(graphs):
            Y.zero_()
            y.zero_()
            ws.fill_(255)
            g.replay()
            assert torch.equal(call(prc, cs[1 - i]), want[1 - i])
            torch.cuda.synchronize()
            assert torch.equal(Y, want[i]) and torch.equal(y, wy) and torch.equal(out, ws_), (rep, i)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("T", [8, 300])
def test_what_a_call_allocates_belongs_to_its_stream(T, raw):
    """Memory that pending work of the current stream still writes is not handed to a call on another stream."""
    c, nrm = project_case(T, T, 512, 528, 4, 16, "mixed"), norm_case(T, 512, True)
    want, (wy, wr) = call(prc, c), prc.add_rms_norm(*nrm)
    size = prc.adapted_projection_workspace_size(T, 512, 528, 4, 16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    bufs = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (size, 2 * T * 528, 2 * T * 512, 2 * T * 512)]
    torch.cuda._sleep(20_000_000)
    for b in bufs:
        b.fill_(255)
    del bufs, b
    st = side.cuda_stream if raw else side
    got = call(prc, c, stream=st)
    y, r = prc.add_rms_norm(*nrm, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(y, wy) and torch.equal(r, wr)


def test_native_and_python_marshalling_agree(monkeypatch):
    from paper_2609_34054_amd import binding
    c, c8 = project_case(9, 20, 256, 272, 3, 16), project_case(9, 20, 256, 272, 3, 16, fp8=True)
    x, w, res = norm_case(20, 256, True)
    calls = [lambda: (call(prc, c),), lambda: (call(prc, c8),), lambda: prc.add_rms_norm(x, w, res),
             lambda: prc.add_rms_norm_fp8(x, w, res), lambda: prc.add_rms_norm(x, w),
             lambda: (call(prc, dict(c, A_stack=None, B=None, agent=None)),)]
    want = [f() for f in calls]
    with monkeypatch.context() as m:
        m.setattr(binding, "_on_gpu", lambda t: False)
        for f, u in zip(calls, want):
            for a, b in zip(f(), u):
                assert (a is None and b is None) or torch.equal(a.float(), b.float())
    # Calls that are not plain come back to the checks that raise.
    for bad, err in ((dict(c, agent=c["agent"].long()), TypeError), (dict(c, X=c["X"].float()), TypeError),
                     (dict(c, W=c["W"].t()), ValueError), (dict(c, B=c["B"][:2]), ValueError),
                     (dict(c, agent=c["agent"].cpu()), ValueError), (dict(c, agent=None), ValueError),
                     (dict(c, A_stack=c["A_stack"].cpu()), ValueError)):
        with pytest.raises(err):
            call(prc, bad)
    with pytest.raises(ValueError):
        prc.add_rms_norm(x, w.cpu(), res)
    with pytest.raises(prc.PrecacheError):   # Y over X
        call(prc, dict(c, W=c["W"][:, :256].contiguous(), B=c["B"][:, :, :256].contiguous()), Y=c["X"])


def test_a_layers_input_to_attention():
    """The operators together as a layer runs them: norm, K/V and LR rows, q with each agent's adapter, attention over
    the shared cache, and o; in bf16 and with the norm and the projections in 8 bits, against the same steps in 64
    bits fed with what the library wrote at each step."""
    T, hid, n_q, n_kv, d, N, r = 96, 512, 8, 2, 64, 3, 16
    rnd = Draws(77)
    x, res, w = rnd.bf16(T, hid), rnd.bf16(T, hid, std=3.0), (1 + rnd(hid, std=0.1)).to(BF)
    Wq, Wkv, Wo = (rnd.bf16(hid, n, std=hid ** -0.5) for n in (n_q * d, 2 * n_kv * d, hid))
    A, Bq = rnd.bf16(hid, N * r, std=hid ** -0.5), rnd.bf16(N, r, n_q * d, std=0.14)
    Ao, Bo = rnd.bf16(n_q * d, N * r, std=(n_q * d) ** -0.5), rnd.bf16(N, r, hid, std=0.14)
    A_kv, Bkv = rnd.bf16(hid, 2 * N * r, std=hid ** -0.5), rnd.bf16(N, 2, r, n_kv * d, std=0.14)
    K, V = (torch.zeros((T, n_kv, d), dtype=BF, device="cuda") for _ in range(2))
    L = torch.zeros((2, N, T, r), dtype=BF, device="cuda")
    y, s = prc.add_rms_norm(x, w, res)
    check_norm(y, x, w, res, 1e-5, s)
    prc.project_kv_and_lr_cache(y, Wkv, A_kv, n_kv, d, 2, N, r, K, V, L, rope_theta=1e4)
    # Three agents ask about the same prefix with its last token each: their rows of q, their own adapters.
    last = y[T - 1:].expand(N, hid).contiguous()
    agent = torch.arange(N, dtype=torch.int32, device="cuda")
    q = prc.adapted_projection(last, Wq, A, Bq, agent)
    check_project(q, *ref_of({"X": last, "W": Wq, "A_stack": A, "B": Bq, "agent": agent}))
    pos = torch.full((N, 1), T - 1, dtype=torch.int32, device="cuda")
    kvl = torch.full((N,), T, dtype=torch.int32, device="cuda")
    O, _ = prc.lr_shared_attention(q.view(N, 1, n_q, d), K[None], V[None], L[0], L[1], Bkv[:, 0].contiguous(),
                                   Bkv[:, 1].contiguous(), pos, kvl, rope_theta=1e4)
    import oracle
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    want, _ = oracle.lr_shared_attention(f(q.view(N, 1, n_q, d)), f(K.expand(N, T, n_kv, d)), f(V.expand(N, T, n_kv, d)), f(L[0]), f(L[1]), f(Bkv[:, 0]),
                                         f(Bkv[:, 1]), pos.cpu().numpy(), kvl.cpu().numpy(), 1e4)
    assert (O.double().cpu() - torch.from_numpy(want)).abs().max() <= 2e-2
    o_in = O.view(N, n_q * d)
    o = prc.adapted_projection(o_in, Wo, Ao, Bo, agent)
    check_project(o, *ref_of({"X": o_in, "W": Wo, "A_stack": Ao, "B": Bo, "agent": agent}))
    # The next norm adds o to the residual, in 8 bits for an 8-bit projection.
    q8, qs, s2 = prc.add_rms_norm_fp8(o, w, s[T - 1:].expand(N, hid).contiguous())
    check_norm_fp8(q8, qs, o, w, s[T - 1:].expand(N, hid), 1e-5, s2)
    from layer_input_ref import quantised
    W8, w8s = quantised(Wq.float(), 0)
    got = prc.adapted_projection_fp8(q8, qs, W8, w8s, A, Bq, agent)
    check_project(got, *ref_of({"X": q8, "x_scale": qs, "W": W8, "w_scale": w8s, "A_stack": A, "B": Bq, "agent": agent}))
    assert q8.dtype == E4M3 and norm_ref(o, w, s2, 1e-5)[0].shape == got.shape[:1] + (hid,)


@pytest.mark.parametrize("T", [3, 700])
def test_checked_library_reports_agents(T):
    from paper_2609_34054_amd.binding import use_checked_library
    c = project_case(4, T, 256, 272, 3, 16, "mixed")
    want = call(prc, c)
    c["agent"][1] = -7
    base = call(prc, c)
    try:
        use_checked_library(True)
        assert torch.equal(call(prc, c), base) and torch.equal(base[2:], want[2:])
        c["agent"][2] = 3
        with pytest.raises(prc.PrecacheError) as e:
            call(prc, c)
        assert e.value.status_name == "PRC_EDEVDATA" and "agent[2]=3" in str(e.value)
    finally:
        use_checked_library(False)
    got = call(prc, c)
    assert torch.equal(got[3:], want[3:]) and torch.isfinite(got.float()).all()
