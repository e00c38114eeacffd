"""Cases of the layer-input operators: the residual sum with its RMS norm, and projections whose rows carry the
low-rank adapters of many agents at once, each in bf16 and in 8 bits (e4m3 with fp32 scales).

Sizes are those of the repository's workloads: a tiny layer (hidden 256), the 8B-shaped layer (hidden 4096, ranks 8 and
16) and the 14B-shaped one (hidden 5120, rank 64), with row counts from one decoded token to a 4096-token segment.

Kinds of case:
  norm     s = x + residual, y = s / rms(s) * weight, per row; "fp8" writes y in e4m3 with one scale a row
  project  Y[i] = X[i] W + (X[i] A_a) B_a with a = agent[i] (a < 0: the base projection alone); "fp8" takes X and W in
           e4m3 with a scale per row of X and per column of W
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
E4M3_MAX = 448.0
TINY = 2.0 ** -100          # least row maximum an 8-bit scale is made from
B_STD = math.sqrt(0.02)     # up-projection entries: N(0, 0.02)
HIDDEN = {"tiny": 256, "8b": 4096, "14b": 5120}


def listed():
    return [
        # One decoded token enters a layer: launch and host time are all there is.
        {"name": "norm_1", "kind": "norm", "T": 1, "d": 4096, "residual": True, "fp8": False, "pad": 0},
        # A decode batch of sixteen requests, its layer input in 8 bits.
        {"name": "norm_16_fp8", "kind": "norm", "T": 16, "d": 4096, "residual": True, "fp8": True, "pad": 0},
        # The first norm of a short chunk (no residual yet), an odd number of rows out of a wider buffer.
        {"name": "norm_333_first", "kind": "norm", "T": 333, "d": 256, "residual": False, "fp8": False, "pad": 64},
        # A long new segment, in bf16 and (wider layer) in 8 bits.
        {"name": "norm_4096", "kind": "norm", "T": 4096, "d": 4096, "residual": True, "fp8": False, "pad": 0},
        {"name": "norm_2048_fp8", "kind": "norm", "T": 2048, "d": 5120, "residual": True, "fp8": True, "pad": 0},
        # q_proj (or o_proj) of one decoded token of one agent.
        {"name": "project_1", "kind": "project", "T": 1, "d_in": 4096, "d_out": 4096, "agents": 8, "rank": 16,
         "order": "mixed", "requests": 1, "base": False, "fp8": False, "pad": 0},
        # A decode batch of sixteen requests of eight agents, every row with its own adapter.
        {"name": "project_16_mixed", "kind": "project", "T": 16, "d_in": 4096, "d_out": 4096, "agents": 8, "rank": 16,
         "order": "mixed", "requests": 1, "base": False, "fp8": False, "pad": 0},
        # The 14B-shaped layer's decode batch in 8 bits, rank-64 adapters.
        {"name": "project_8_fp8_r64", "kind": "project", "T": 8, "d_in": 5120, "d_out": 5120, "agents": 6, "rank": 64,
         "order": "mixed", "requests": 1, "base": False, "fp8": True, "pad": 0},
        # One agent's prompt chunk.
        {"name": "project_512", "kind": "project", "T": 512, "d_in": 4096, "d_out": 4096, "agents": 4, "rank": 16,
         "order": "runs", "requests": 1, "base": False, "fp8": False, "pad": 0},
        # A ragged batch of chunks of five requests, one of them the base model's.
        {"name": "project_1000_ragged", "kind": "project", "T": 1000, "d_in": 4096, "d_out": 4096, "agents": 8,
         "rank": 8, "order": "runs", "requests": 5, "base": True, "fp8": False, "pad": 64},
        # The largest: a long segment cut between three requests.
        {"name": "project_4096", "kind": "project", "T": 4096, "d_in": 4096, "d_out": 4096, "agents": 8, "rank": 16,
         "order": "runs", "requests": 3, "base": False, "fp8": False, "pad": 0},
        # The 14B-shaped layer's chunk in 8 bits.
        {"name": "project_2048_fp8_r64", "kind": "project", "T": 2048, "d_in": 5120, "d_out": 5120, "agents": 6,
         "rank": 64, "order": "runs", "requests": 2, "base": False, "fp8": True, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    fp8 = rng.random() < 0.4
    step = 16
    pad = rng.choice([0, 0, 0, 64, 16])

    def width():
        return rng.choice([HIDDEN["tiny"], HIDDEN["8b"], HIDDEN["8b"], HIDDEN["14b"],
                           step * _log_int(rng, 256 // step, 8192 // step)])

    if rng.random() < 0.35:
        return {"kind": "norm", "T": _log_int(rng, 1, 4096), "d": width(), "residual": rng.random() < 0.8, "fp8": fp8,
                "pad": pad}
    c = {"kind": "project", "T": _log_int(rng, 1, 4096), "d_in": width(), "d_out": width(),
         "agents": rng.choice([1, 3, 4, 6, 8, 8, 32]), "rank": rng.choice([8, 16, 16, 32, 64]),
         "order": rng.choice(["runs", "runs", "mixed"]), "requests": rng.randint(1, 8), "base": rng.random() < 0.3,
         "fp8": fp8, "pad": pad}
    c["requests"] = min(c["requests"], c["T"])
    # No dearer than the largest listed one.
    while c["T"] * c["d_in"] * c["d_out"] > 4096 ** 3:
        c["T"] = c["T"] * 3 // 4
    return c


def _agents_used(c):
    """Distinct adapters that the rows of a case use (of mixed rows: all that there is room for)."""
    n = c["requests"] - (1 if c["base"] else 0) if c["order"] == "runs" else c["T"]
    return min(c["agents"], max(n, 0))


def work(case):
    c = case
    T = c["T"]
    if c["kind"] == "norm":
        d = c["d"]
        per = 2 + (4 if c["residual"] else 0) + (1 if c["fp8"] else 2)
        return {"bytes": T * d * per + 2 * d + (4 * T if c["fp8"] else 0), "flops": 8 * T * d}
    k, n, r, e = c["d_in"], c["d_out"], c["rank"], 1 if c["fp8"] else 2
    return {"bytes": e * (T * k + k * n) + 2 * T * n + 2 * _agents_used(c) * r * (k + n) + 4 * T
            + (4 * (T + n) if c["fp8"] else 0),
            "flops": 2 * T * k * n + 2 * T * r * (k + n)}


def _agent_rows(c, g):
    """The adapter of every row, on the host: runs of ragged length (one request each), or every row its own."""
    T, N = c["T"], c["agents"]
    if c["order"] == "mixed":
        a = torch.randint(0, N, (T,), generator=g)
        if c["base"]:
            a[torch.rand(T, generator=g) < 0.2] = -1
        return a.to(torch.int32)
    n = min(c["requests"], T)
    cuts = torch.cat([torch.zeros(1, dtype=torch.long), 1 + torch.randperm(T - 1, generator=g)[:n - 1].sort().values])
    run = torch.bucketize(torch.arange(T), cuts, right=True) - 1
    a = (run + torch.randint(0, N, (1,), generator=g)) % N
    if c["base"]:
        a[run == n - 1] = -1
    return a.to(torch.int32)


def _quantised(x, dim):
    """x in e4m3 with fp32 scales over `dim`."""
    scale = x.abs().amax(dim).clamp_min(TINY) / E4M3_MAX
    return (x / scale.unsqueeze(dim)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))

    def rnd(*shape, std=1.0):
        return torch.randn(shape, generator=g, dtype=torch.float32, device="cuda").mul_(std)

    def rows(x):
        """x as rows of a wider buffer."""
        if not c["pad"]:
            return x
        wide = torch.zeros((x.shape[0], x.shape[1] + c["pad"]), dtype=x.dtype, device="cuda")
        wide[:, :x.shape[1]] = x
        return wide[:, :x.shape[1]]

    s = {"case": c}
    T = c["T"]
    bf = torch.bfloat16
    if c["kind"] == "norm":
        d = c["d"]
        s["x"] = rows(rnd(T, d).to(bf))
        s["weight"] = (1.0 + rnd(d, std=0.1)).to(bf)
        s["residual"] = None
        if c["residual"]:
            # A residual stream: larger than a layer's output, with a few channels far larger.
            gain = torch.full((d,), 3.0, device="cuda")
            gain[torch.randperm(d, generator=host)[:max(1, d // 512)].cuda()] = 60.0
            s["residual"] = rows((rnd(T, d) * gain).to(bf))
        s["residual_out"] = torch.empty((T, d), dtype=bf, device="cuda") if c["residual"] else None
        s["y"] = torch.empty((T, d), dtype=torch.float8_e4m3fn if c["fp8"] else bf, device="cuda")
        s["y_scale"] = torch.empty(T, dtype=torch.float32, device="cuda") if c["fp8"] else None
        return s
    k, n, r, N = c["d_in"], c["d_out"], c["rank"], c["agents"]
    X, W = rnd(T, k), rnd(k, n, std=1 / math.sqrt(k))
    if c["fp8"]:
        X, s["x_scale"] = _quantised(X, 1)
        s["W"], s["w_scale"] = _quantised(W, 0)
        s["X"] = rows(X.view(torch.uint8)).view(torch.float8_e4m3fn)
    else:
        s["X"], s["W"] = rows(X.to(bf)), W.to(bf)
    s["A"] = rnd(k, N * r, std=1 / math.sqrt(k)).to(bf)
    s["B"] = rnd(N, r, n, std=B_STD).to(bf)
    s["agent"] = _agent_rows(c, host).cuda()
    s["Y"] = torch.empty((T, n), dtype=bf, device="cuda")
    # The scratch memory that a serving loop keeps for all its projections.
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    import paper_2609_34054_amd as prc
    c = s["case"]
    if c["kind"] == "norm":
        if c["fp8"]:
            y, scale, out = prc.add_rms_norm_fp8(s["x"], s["weight"], s["residual"], eps=EPS, y=s["y"],
                                                 y_scale=s["y_scale"], residual_out=s["residual_out"])
            return {"y": y, "scale": scale, "residual": out}
        y, out = prc.add_rms_norm(s["x"], s["weight"], s["residual"], eps=EPS, y=s["y"],
                                  residual_out=s["residual_out"])
        return {"y": y, "residual": out}
    if c["fp8"]:
        return prc.adapted_projection_fp8(s["X"], s["x_scale"], s["W"], s["w_scale"], s["A"], s["B"], s["agent"],
                                          Y=s["Y"], workspace=s["workspace"])
    return prc.adapted_projection(s["X"], s["W"], s["A"], s["B"], s["agent"], Y=s["Y"], workspace=s["workspace"])


def run(state):
    if own:
        return _run_own(state)
    s = state
    c = s["case"]
    if c["kind"] == "norm":
        v = s["x"].float()
        out = None
        if c["residual"]:
            v = v + s["residual"].float()
            out = v.to(torch.bfloat16)
        z = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * s["weight"].float()
        if not c["fp8"]:
            return {"y": z.to(torch.bfloat16), "residual": out}
        scale = z.abs().amax(-1).clamp_min(TINY) / E4M3_MAX
        q = (z / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return {"y": q, "scale": scale, "residual": out}
    T, N, r = c["T"], c["agents"], c["rank"]
    X, W = s["X"].float(), s["W"].float()
    if c["fp8"]:
        X, W = X * s["x_scale"][:, None], W * s["w_scale"][None, :]
    mine = s["agent"][:, None] == torch.arange(N, dtype=torch.int32, device="cuda")[None, :]
    H = (X @ s["A"].float()).view(T, N, r) * mine[:, :, None]
    return (X @ W + H.view(T, N * r) @ s["B"].float().view(N * r, -1)).to(torch.bfloat16)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "norm":
        v = s["x"].double()
        if c["residual"]:
            v += s["residual"].double()
        z = v / torch.sqrt(v.square().sum(1, keepdim=True) / c["d"] + EPS) * s["weight"].double()
        out = v if c["residual"] else None
        if not c["fp8"]:
            return {"y": z, "residual": out}
        scale = z.abs().max(1).values / E4M3_MAX
        # The values of y before their rounding to 8 bits.
        return {"y": z / scale[:, None], "scale": scale, "residual": out}
    X, W = s["X"].to(torch.float64), s["W"].to(torch.float64)
    if c["fp8"]:
        X, W = X * s["x_scale"].double()[:, None], W * s["w_scale"].double()[None, :]
    Y, r = X @ W, c["rank"]
    for a in range(c["agents"]):
        i = (s["agent"] == a).nonzero().flatten()
        if len(i):
            Y[i] += X[i] @ s["A"][:, a * r:(a + 1) * r].double() @ s["B"][a].double()
    return Y
