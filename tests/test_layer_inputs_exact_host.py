"""What the exact projection cases notice, on the host: the mistakes are made in the plain 64-bit form."""
import pytest
import torch

from layer_input_exact import BF, exact_case, exact_y

CASES = [(5, 264, 72, 3, 8, False), (5, 272, 144, 3, 8, True), (33, 4112, 64, 2, 16, False), (20, 8, 40, 4, 64, False),
         (17, 16, 48, 4, 32, True), (9, 65536, 64, 2, 16, False), (9, 65536, 64, 2, 16, True)]


@pytest.mark.parametrize("T,k,n,N,r,fp8", CASES)
def test_results_are_numbers_of_bf16(T, k, n, N, r, fp8):
    for wide in (False, True):
        y = exact_y(exact_case(T + k, T, k, n, N, r, fp8, wide, "cpu"))
        assert torch.equal(y.to(BF).double(), y)


@pytest.mark.parametrize("T,k,n,N,r,fp8", CASES)
def test_lost_k_and_adapters_show(T, k, n, N, r, fp8):
    c = exact_case(T + k, T, k, n, N, r, fp8, False, "cpu")
    y = exact_y(c)
    last = torch.ones(k)
    last[k - 8:] = 0
    assert (exact_y(c, keep=last) != y).any(1).all()
    assert ((exact_y(c, adapters=False) != y).any(1) == (c["agent"] >= 0)).all()
    for parts in (2, 3, 8, 16):   # a slice of k: of many, one that no row of a short case uses may be lost
        for i in range(parts):
            keep = torch.ones(k)
            keep[k * i // parts:k * (i + 1) // parts] = 0
            used = (c["X"].double() * (1 - keep)).abs().sum(1) > 0
            assert (exact_y(c, keep=keep) != y)[used].any(1).all() and (used.any() or k < 16 * parts)


@pytest.mark.parametrize("T,k,n,N,r,fp8", CASES)
def test_rows_of_fewer_bits_show(T, k, n, N, r, fp8):
    c = exact_case(T + k, T, k, n, N, r, fp8, True, "cpu")
    assert k < 32 or ((exact_y(c, bf16_rows=True) != exact_y(c)).any(1) == (c["agent"] >= 0)).all()
