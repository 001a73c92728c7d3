"""All rows with one expert of many: its gradient's tile is one CTA's work for longer than any wait's limit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
ROWS = 500_000_037


@pytest.mark.parametrize("gather", [False, True])
def test_dw_of_a_contraction_that_takes_long(gather):
    from paper_2608_27888_gb300 import ntc
    E, K, N, e = 100, 8, 8, 41
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[e + 1:] = ROWS
    w = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros(ROWS, N, dtype=torch.bfloat16, device="cuda")
    # small whole numbers, so that every sum is exact: both ends, and rows spread over the rest
    at = torch.cat([torch.arange(70), torch.arange(10_007, ROWS - 100, 20_000_003), torch.arange(ROWS - 70, ROWS)]).cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    dy[at] = torch.randint(-3, 4, (at.numel(), N), generator=g, device="cuda").bfloat16()
    some = torch.randint(-2, 3, (at.numel(), K), generator=g, device="cuda").bfloat16()
    if gather:
        x, rows = torch.cat([torch.zeros_like(some[:1]), some]), torch.zeros(ROWS, dtype=torch.int32, device="cuda")
        rows[at] = torch.arange(1, at.numel() + 1, dtype=torch.int32, device="cuda")
    else:
        x, rows = torch.zeros(ROWS, K, dtype=torch.bfloat16, device="cuda"), None
        x[at] = some
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    _, dw, _ = ntc.linear_backward(dy, x, w, rows=rows, offsets=offsets, need=("dw",))
    end.record()
    want = torch.zeros(E, N, K, dtype=torch.float64, device="cuda")
    want[e] = dy[at].double().T @ some.double()
    assert torch.equal(dw, want.bfloat16())
    ntc.ntc_linear_status(torch.cuda.current_stream().cuda_stream)
    assert start.elapsed_time(end) > 200  # what the test is about: past the limit of one wait
    del x, dy, rows
    torch.cuda.empty_cache()
