"""Adapted projections of whole numbers, whose results are exact: compared bit for bit."""
import pytest
import torch

from layer_input_exact import exact_case, exact_y
from layer_input_ref import call
import paper_2609_34054_amd as prc

pytestmark = pytest.mark.gpu

# One of each form and tile shape: rows streamed, slabs, tiles of 128 x 64 to 256 x 256; ends inside tiles.
FORMS = [(1, 1032, 264), (16, 528, 144), (40, 1040, 272), (100, 2064, 1040), (1000, 1024, 4096), (2500, 1040, 2064),
         (2040, 272, 5120), (2040, 528, 6144), (4090, 272, 4080), (3000, 528, 4096)]


def check(c):
    got, want = call(prc, c), exact_y(c)
    wrong = (got.double() != want).nonzero()
    assert not len(wrong), (len(wrong), wrong[0].tolist(), float(got[tuple(wrong[0])]), float(want[tuple(wrong[0])]))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n", FORMS)
def test_adapter_rows_keep_their_bits(T, k, n, fp8):
    """Entries of X A_a of 14 bits that cancel in Y."""
    k, n = ((k + 15) // 16 * 16, (n + 15) // 16 * 16) if fp8 else (k, n)
    for r, N in ((8, 3), (16, 1), (32, 12), (64, 9)):
        print(f"project {T} {k} {n} {N} r{r} fp8={fp8}", flush=True)
        check(exact_case(T + k + r, T, k, n, N, r, fp8, wide=True))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [3, 40, 1000])
def test_an_infinite_adapter_row_is_infinite(T, fp8):
    """Not NaN: a row of X A_a that is infinite, times one."""
    c = exact_case(T, T, 1024, 4096, 2, 16, fp8, device="cuda")
    c["agent"].fill_(1)
    c["B"].zero_()
    c["B"][1] = 1.0
    c["A_stack"][1023, 16 + 5] = float("inf")   # X is 1 there in every row
    assert (call(prc, c) == float("inf")).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n,N,r", [
    (1, 65536, 64, 2, 16), (3, 8192, 1024, 3, 32), (9, 65552, 144, 4, 64), (16, 32784, 272, 5, 8), (17, 65536, 64, 2, 16),
    (40, 65488, 80, 3, 64), (130, 65536, 64, 2, 8), (640, 65536, 64, 2, 16), (700, 32784, 2064, 3, 32), (2500, 16400, 2064, 9, 64),
    (4097, 32768, 256, 1, 16), (20, 1 << 21, 16, 1, 8), (70, 1 << 20, 32, 1, 16),
])
def test_long_sums_leave_nothing_out(T, k, n, N, r, fp8):
    """Every slice of a long k, its end and the adapters: a bound on the roundings of a sum would hide them."""
    print(f"project {T} {k} {n} {N} r{r} fp8={fp8}", flush=True)
    for seed in range(3 if T < 32 else 1):
        check(exact_case(T + k + r + seed, T, k, n, N, r, fp8))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n", FORMS)
def test_projections_of_whole_numbers(T, k, n, fp8):
    k, n = ((k + 15) // 16 * 16, (n + 15) // 16 * 16) if fp8 else (k, n)
    for r, N in ((8, 12), (64, 3)):
        check(exact_case(T + k + r, T, k, n, N, r, fp8))


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("T,k,n", FORMS)
def test_scales_and_agents_off_16_byte_lines(T, k, n, off):
    """fp32 and int32 arrays need 4-byte alignment alone."""
    k, n = (k + 15) // 16 * 16, (n + 15) // 16 * 16
    c = exact_case(T + off, T, k, n, 3, 16, fp8=True)
    for name in ("x_scale", "w_scale", "agent"):
        wide = torch.zeros(len(c[name]) + 8, dtype=c[name].dtype, device="cuda")
        wide[off:off + len(c[name])] = c[name]
        c[name] = wide[off:off + len(c[name])]
        assert c[name].data_ptr() % 16 == 4 * off
    check(c)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,k,n", FORMS)
def test_nothing_is_written_past_the_workspace_and_the_rows(T, k, n, fp8):
    k, n = ((k + 15) // 16 * 16, (n + 15) // 16 * 16) if fp8 else (k, n)
    for r, N in ((8, 12), (64, 3)):
        c = exact_case(T + k + r, T, k, n, N, r, fp8)
        size = prc.adapted_projection_workspace_size(T, k, n, N, r)
        ws = torch.full((size + 4096,), 90, dtype=torch.uint8, device="cuda")
        Y = torch.full((T + 5, n + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        call(prc, c, Y=Y[2:T + 2, :n], workspace=ws[:size])
        assert torch.all(ws[size:] == 90)
        assert torch.equal(Y[2:T + 2, :n].double(), exact_y(c))
        assert torch.all(Y[:2] == 7.0) and torch.all(Y[T + 2:] == 7.0) and torch.all(Y[:, n:] == 7.0)


def test_checked_calls_of_two_threads_read_their_own_verdicts():
    """One thread's agents past the last, another's valid ones, each on its own stream: none takes the other's."""
    from concurrent.futures import ThreadPoolExecutor
    from paper_2609_34054_amd.binding import use_checked_library
    good, bad = (exact_case(i, 20, 256, 272, 3, 16) for i in range(2))
    bad["agent"][7] = 3
    want = exact_y(good)

    def run(c, stream):
        seen = []
        with torch.cuda.stream(stream):
            for _ in range(200):
                try:
                    seen.append(call(prc, c))
                except prc.PrecacheError as e:
                    seen.append(e)
            stream.synchronize()
        return seen

    torch.cuda.synchronize()
    use_checked_library(True)
    try:
        with ThreadPoolExecutor(2) as pool:
            goods, bads = (f.result() for f in [pool.submit(run, c, torch.cuda.Stream()) for c in (good, bad)])
    finally:
        use_checked_library(False)
    assert all(isinstance(e, prc.PrecacheError) and e.status_name == "PRC_EDEVDATA" and "agent[7]=3" in str(e) for e in bads)
    assert all(torch.equal(y.double(), want) for y in goods)
