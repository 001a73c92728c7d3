"""The routed experts' operators where elements lie past 2^31 and bytes past 2^32.

Exact or against 64 bits at both ends of the long tensors.  The products' inputs are
small integers, so that every sum is exact in fp32 and the results are what 64 bits
give, rounded once.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS = (1 << 20) + 37  # of 2,048 elements: past 2^31 of them


def whole(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    yield ntc
    torch.cuda.empty_cache()


ENDS = (slice(0, 300), slice(ROWS - 300, ROWS))


def test_a_long_result_and_its_gradients(ntc):
    x, w = whole((ROWS, 64), 1), whole((2048, 64), 2)
    y = ntc.linear(x, w)
    for s in ENDS:
        assert torch.equal(y[s], (x[s].double() @ w.double().T).to(y.dtype))
    # a gradient of zeros but for both ends: sums that are exact
    y.zero_()
    for i, s in enumerate(ENDS):
        y[s] = whole((300, 2048), 3 + i)
    dx, dw, db = ntc.linear_backward(y, x, w)
    for s in ENDS:
        assert torch.equal(dx[s], (y[s].double() @ w.double()).to(dx.dtype))
    assert int(dx[300:ROWS - 300].abs().max()) == 0
    assert torch.equal(dw, sum(y[s].double().T @ x[s].double() for s in ENDS).to(dw.dtype))
    assert torch.equal(db.double(), sum(y[s].double().sum(0) for s in ENDS))
    ntc.ntc_linear_status(0)


@pytest.mark.parametrize("rows", [12, 700])
def test_rows_and_weights_far_into_their_tensors(ntc, rows):
    E, K, N = 600, 2048, 2048  # weights: 2.5e9 elements
    x = torch.empty((ROWS, K), dtype=torch.bfloat16, device="cuda")
    w = torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
    far = torch.arange(ROWS - rows, ROWS, dtype=torch.int32, device="cuda").flip(0).contiguous()
    x[ROWS - rows:] = whole((rows, K), 5)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    half = rows // 2
    offsets[1:] = half
    offsets[E] = rows
    for i, e in enumerate((0, E - 1)):
        w[e] = whole((N, K), 6 + i)
    y = ntc.linear(x, w, rows=far, offsets=offsets)
    ours = x[far.long()].double()
    want = torch.cat([ours[:half] @ w[0].double().T, ours[half:] @ w[E - 1].double().T])
    assert torch.equal(y, want.to(y.dtype))
    ntc.ntc_linear_status(0)


def test_a_long_blend_and_its_gradient(ntc):
    y = torch.zeros((ROWS, 2048), dtype=torch.bfloat16, device="cuda")
    for i, s in enumerate(ENDS):
        y[s] = whole((300, 2048), 8 + i)
    place = torch.arange(ROWS, dtype=torch.int32, device="cuda").flip(0).reshape(ROWS, 1).contiguous()
    weights = torch.full((ROWS, 1), 0.5, device="cuda")
    out = ntc.combine(y, place, weights)
    for s in ENDS:
        assert torch.equal(out[s], y.flip(0)[s] * 0.5)
    dy, dweights = ntc.combine_backward(out, y, place, weights)
    for s in ENDS:
        assert torch.equal(dy[s], out.flip(0)[s] * 0.5)
        want = (out[s].double() * y.flip(0)[s].double()).sum(1)
        # multiples of a half, sums below 2^13: exact
        assert torch.equal(dweights[s].flatten().double(), want)


def test_routing_of_many_tokens(ntc):
    T, E = (1 << 23) + 11, 256  # 2.1e9 logits
    logits = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(10)
    end = torch.randn((500, E), generator=g, device="cuda").bfloat16()
    logits[T - 500:] = end
    ids, weights = ntc.route(logits, 4)[:2]
    some_ids, some_weights = ntc.route(end.contiguous(), 4)[:2]
    assert torch.equal(ids[T - 500:], some_ids) and torch.equal(weights[T - 500:], some_weights)
    assert torch.equal(ids[:1000], torch.arange(4, dtype=torch.int32, device="cuda").expand(1000, 4))
