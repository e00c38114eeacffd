"""What the exact projection cases notice, on the host: the mistakes are made in the plain 64-bit form."""
import contextlib

import pytest
import torch

import paper_2609_34054_amd as prc
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
    for parts in (2, 3, 8, 16):   # a slice of k (of a short k, one that no row uses may be lost)
        for i in range(parts):
            keep = torch.ones(k)
            keep[k * i // parts:k * (i + 1) // parts] = 0
            used = (c["X"].double() * (1 - keep)).abs().sum(1) > 0
            assert (exact_y(c, keep=keep) != y)[used].any(1).all() and (used.all() or k < 16 * parts or parts == 16)


@pytest.mark.parametrize("T,k,n,N,r,fp8", CASES)
def test_rows_of_fewer_bits_show(T, k, n, N, r, fp8):
    c = exact_case(T + k, T, k, n, N, r, fp8, True, "cpu")
    assert k < 32 or ((exact_y(c, bf16_rows=True) != exact_y(c)).any(1) == (c["agent"] >= 0)).all()


def test_a_raw_stream_is_taken_for_one_of_the_tensors_device(monkeypatch):
    """What a call allocates for a raw stream handle belongs to that stream of the tensors' device, which need not be
    the current one.  (Tensors of the host, which the calls then refuse.)"""
    devices = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=None: devices.append((ptr, device)))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    c = exact_case(1, 6, 64, 32, 3, 8, device="cpu")
    with pytest.raises(ValueError, match="not on a GPU"):
        prc.adapted_projection(c["X"], c["W"], c["A_stack"], c["B"], c["agent"], stream=4096)
    with pytest.raises(ValueError, match="not on a GPU"):
        prc.add_rms_norm(c["X"], torch.ones(64, dtype=BF), c["X"], stream=4096)
    assert devices and set(devices) == {(4096, c["X"].device)}
