"""A layer's attention half from its hidden states, q's rotation by the caller among the steps, against the layer's
definition in 64 bits (the oracle, fed with the hidden states and the weights alone)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_34054_amd as prc
from layer_input_ref import Draws

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
T, HID, N_Q, N_KV, D, N, R, THETA = 96, 512, 8, 2, 64, 3, 16, 1e4

# Roundings to bf16 between the hidden states and a score, half a step (2^-8, a standard deviation of 2^-8 / sqrt(3) at
# most) each: q twice (projection, rotation), K, L, the rebuilt key, the probability.  A score's products have a root
# sum of squares of about 1 over sqrt(d), so it is off by sqrt(6) 2^-8 / sqrt(3) = 0.0055, five of them 0.028; the output
# by that times the weighted mean of |V - O|, about 0.9, and half a step of V's part and of the output, 1.5 * 2^-8 each.
TOL = 0.025 + 2 * 1.5 * 2.0 ** -8


def rotated(q, pos):
    """Rotate-half of q [T, n_q, d] at pos [T], as the caller of lr_shared_attention does it."""
    omega = THETA ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=q.device) / D)
    ang = pos.double()[:, None, None] * omega
    lo, hi = q.double().chunk(2, -1)
    return torch.cat([lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()], -1).to(BF)


@pytest.mark.parametrize("n_tok", [1, 40])
def test_query_is_rotated_between_projection_and_attention(n_tok):
    rnd = Draws(78)
    y = rnd.bf16(T, HID)
    Wq, Wkv = rnd.bf16(HID, N_Q * D, std=HID ** -0.5), rnd.bf16(HID, 2 * N_KV * D, std=HID ** -0.5)
    A, Bq = rnd.bf16(HID, N * R, std=HID ** -0.5), rnd.bf16(N, R, N_Q * D, std=0.14)
    A_kv = rnd.bf16(HID, 2 * N * R, std=HID ** -0.5)
    B_k, B_v = rnd.bf16(N, R, N_KV * D, std=0.14), rnd.bf16(N, R, N_KV * D, std=0.14)
    K, V = (torch.zeros((T, N_KV, D), dtype=BF, device="cuda") for _ in range(2))
    L = torch.zeros((2, N, T, R), dtype=BF, device="cuda")
    prc.project_kv_and_lr_cache(y, Wkv, A_kv, N_KV, D, 2, N, R, K, V, L, rope_theta=THETA)
    # Every agent asks with the segment's last tokens: their rows of q, one after another, its own adapter.
    rows = torch.arange(T - n_tok, T, device="cuda")
    agent = torch.arange(N, dtype=torch.int32, device="cuda").repeat_interleave(n_tok)
    q = prc.adapted_projection(y[rows].repeat(N, 1), Wq, A, Bq, agent).view(N * n_tok, N_Q, D)
    pos = rows.to(torch.int32).expand(N, n_tok).contiguous()
    kvl = torch.full((N,), T, dtype=torch.int32, device="cuda")
    O, _ = prc.lr_shared_attention(rotated(q, pos.flatten()).view(N, n_tok, N_Q, D), K[None], V[None], L[0], L[1], B_k, B_v,
                                   pos, kvl, rope_theta=THETA)

    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    p = np.arange(T - n_tok, T)
    K64, V64, L64 = oracle.project_kv_and_lr(f(y), f(Wkv[:, :N_KV * D]), f(Wkv[:, N_KV * D:]), f(A_kv), N_KV, 2, N, R,
                                             np.arange(T), THETA)
    for a in range(N):
        q64 = f(y)[p] @ f(Wq) + f(y)[p] @ f(A)[:, a * R:(a + 1) * R] @ f(Bq)[a]
        q64 = q64.reshape(n_tok, N_Q, D)
        want, plain = (oracle.lr_shared_attention(x[None], K64[None], V64[None], L64[0, a][None], L64[1, a][None],
                                                  f(B_k)[a][None], f(B_v)[a][None], p[None], [T], THETA)[0][0]
                       for x in (oracle.rope(q64, p[:, None], THETA), q64))
        assert np.abs(f(O[a]) - want).max() <= TOL
        assert np.abs(plain - want).max() >= 10 * TOL   # an unrotated q would show
