"""linear4 rounds no weight: whatever the rows, widths, addresses, type and group, a row's result is the product of the
numbers and scales themselves.

Whole numbers with |x| <= 1 and scales of s / 64, s < S: every sum of any of their products, in any order, is a multiple of
1 / 64 below K * 8 * S / 64, which fp32 holds exactly where K * 8 * S <= 2^24.  So the result is the exact one, rounded
once: equal bits, no tolerance.  A scale times a number has up to 8 + 3 (bf16) or 11 + 3 (fp16) bits, three more than the
type holds."""
import math

import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu
H, B, F = torch.float16, torch.bfloat16, torch.float32
MOST = {H: 2048, B: 256}  # scales below these have the type's bits


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def whole(E, N, K, group, dtype, seed):
    """packed, scales and the weights in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-8, 8, (E, N, K + K % 2), generator=g, device="cuda")
    q[..., K:] = 0
    s = (torch.randint(1, MOST[dtype], (E, N, -(-K // group)), generator=g, device="cuda").double() / 64).to(dtype)
    packed = torch.zeros(E, N, (K + 31) // 32 * 16, dtype=torch.uint8, device="cuda")
    packed[..., :(K + 1) // 2] = ((q[..., 0::2] + 8) | (q[..., 1::2] + 8) << 4).to(torch.uint8)
    return packed[..., :(K + 1) // 2], s, q[..., :K].double() * s.double().repeat_interleave(group, -1)[..., :K], g


def cut(x, dtype, at):
    """x in rows that start `at` elements past 16 bytes; at 0: rows of whole 16 bytes."""
    T, K = x.shape
    big = torch.full((T, (K + at + 7) // 8 * 8), math.nan, dtype=dtype, device="cuda")
    big[:, at:at + K] = x
    return big[:, at:at + K]


def shift(t, fill):
    """t in rows that start on no multiple of anything."""
    big = torch.full(t.shape[:-1] + (t.shape[-1] + 3,), fill, dtype=t.dtype, device="cuda")
    big[..., 1:-2] = t
    return big[..., 1:-2]


# rows, experts, choices, out, in: a few rows, tiles of every size, few tiles and many, rows that take several tiles
SIZES = [(1, 1, 1, 40, 512), (7, 1, 1, 48, 512), (13, 1, 1, 130, 500), (30, 1, 1, 33, 480), (40, 1, 1, 200, 512), (100, 1, 1, 8200, 96),
         (150, 1, 1, 130, 333), (500, 1, 1, 257, 512), (1000, 3, 1, 64, 352), (40, 8, 3, 70, 512), (300, 24, 2, 400, 160),
         (700, 256, 8, 129, 96), (900, 64, 3, 330, 160), (4000, 16, 2, 300, 224), (1500, 33, 2, 257, 128), (2000, 4, 2, 72, 31)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("T,E,k,N,K", SIZES)
def test_no_weight_is_rounded(ntc, T, E, k, N, K, group, dtype):
    packed, scales, w, g = whole(E, N, K, group, dtype, T + N)
    ones = torch.randint(-1, 2, (T, K), generator=g, device="cuda")
    rows = offsets = None
    n = T
    if E > 1:
        ids = torch.rand(T, E, generator=g, device="cuda").topk(k, 1).indices.int()
        ids[::7] = -1
        rows, _, offsets = R.order(ids, E)
        n = T * k
    want = torch.zeros(n, N, dtype=torch.float64, device="cuda")
    xs = R.gathered(ones, rows)
    for e, a, o in R.segments(offsets, n):
        want[a:o] = xs[a:o] @ w[e].t()
    want = want.to(dtype)
    for at in (0, 1):
        x = cut(ones.to(dtype), dtype, at)
        y = ntc.linear4(x, packed, scales, group=group, rows=rows, offsets=offsets)
        assert torch.equal(y, want), at
    y = ntc.linear4(cut(ones.to(dtype), dtype, 0), shift(packed, 255), shift(scales, math.nan), group=group, rows=rows, offsets=offsets)
    assert torch.equal(y, want)


@pytest.mark.parametrize("T,E", [(7, 1), (100, 1), (300, 1), (900, 1), (900, 12), (3000, 64)])
@pytest.mark.parametrize("N,K", [(200, 256), (40, 100), (1024, 128)])
def test_a_scale_times_a_number_may_pass_the_types_largest(ntc, T, E, N, K):
    """fp16 scales up to 65,504: a weight is up to 524,032, and two of them times 2^-11 are a small number."""
    g = torch.Generator(device="cuda").manual_seed(T)
    q = torch.randint(-8, 8, (E, N, K), generator=g, device="cuda")
    s = (torch.randint(1024, 2048, (E, N, -(-K // 32)), generator=g, device="cuda").double() * 32).to(H)
    packed = torch.zeros(E, N, (K + 31) // 32 * 16, dtype=torch.uint8, device="cuda")
    packed[..., :K // 2] = ((q[..., 0::2] + 8) | (q[..., 1::2] + 8) << 4).to(torch.uint8)
    x = torch.zeros(T, K, device="cuda")
    x.scatter_(1, torch.rand(T, K, generator=g, device="cuda").topk(2, 1).indices, 2.0 ** -11)
    offsets = torch.arange(E + 1, device="cuda").mul(T).div(E, rounding_mode="floor").int() if E > 1 else None
    y = ntc.linear4(x.to(H), packed[..., :K // 2], s, group=32, offsets=offsets)
    w = q.double() * s.double().repeat_interleave(32, -1)[..., :K]
    want = torch.cat([x[a:o].double() @ w[e].t() for e, a, o in R.segments(offsets, T)])
    assert torch.equal(y, want.to(H))  # both terms are multiples of 2^-6 below 2^8


@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("K", [256, 771])
def test_a_rows_digits_do_not_depend_on_the_batch(ntc, dtype, K):
    """A row alone and among many, at any address: the sums' order may differ, the weights do not.  A result is off by the
    fp32 sums, K + 8 steps of 2^-23 of the terms' magnitudes, and its own rounding."""
    g = torch.Generator(device="cuda").manual_seed(K)
    w = torch.randn(96, K, generator=g, device="cuda") * K ** -0.5
    packed, scales = ntc.pack4(w, group=64, dtype=dtype)
    v = S.values(packed, scales, K, 64)
    x = torch.randn(700, K, generator=g, device="cuda").to(dtype)
    want, mag = x.double() @ v.t(), x.double().abs() @ v.abs().t()
    for T in (1, 9, 33, 200, 700):
        for at in (0, 3):
            y = ntc.linear4(cut(x[:T], dtype, at), packed, scales, group=64)
            off = mag[:T] * (K + 8) * R.F32
            R.assert_within(y, want[:T], off + R.UNIT[dtype] * (want[:T].abs() + off) + R.TINY[dtype], (T, at))


@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("T", [3, 12, 30, 100, 900])
@pytest.mark.parametrize("K", [128, 100])
def test_an_index_outside_x_reads_zeros_whatever_the_rows(ntc, T, K, dtype):
    """Zeros times a scale that is no number are no number, as in the product with 16-bit weights; elsewhere the bias is left."""
    packed, scales, _, g = whole(1, 70, K, 32, dtype, T)
    scales[0, 7, 1], scales[0, 68, 2] = math.nan, math.inf
    x = torch.full((4, K), math.nan, dtype=dtype, device="cuda")
    x[1:3] = 1.0
    rows = torch.randint(1, 3, (T,), generator=g, device="cuda", dtype=torch.int32)
    rows[::3], rows[1::3] = -1, 4
    bias = torch.randn(70, generator=g, device="cuda")
    y = ntc.linear4(x, packed[0], scales[0], bias, group=32, rows=rows)
    z = ntc.linear(x, ntc.unpack4(packed[0], scales[0], K, group=32), bias, rows=rows)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[7] = bad[68] = True
    for out in (y, z):
        gone = out[(rows < 0) | (rows > 3)]
        assert bool(torch.isnan(gone[:, bad]).all()) and torch.equal(gone[:, ~bad], bias[~bad].to(dtype).expand(gone.shape[0], -1))


@pytest.mark.parametrize("K", [96, 97])
def test_copied_operands_with_offsets_that_are_anything(ntc, K):
    """Operands at odd addresses are copied for the experts that have rows, whatever the offsets: the same bits as in order."""
    T, E, N = 400, 5, 40
    packed, scales, _, g = whole(E, N, K, 32, B, K)
    x = torch.randn(T, K, generator=g, device="cuda").to(B)
    rows = torch.randint(-1, T + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    for o in ([0, 0, 2, 1, 4, T], [-5, 3, 3, 3, 4, 10 * T], [T] * 6, [0] * 6, [2, 1, 0, 3, 2, T // 2], [-2 ** 31, 2 ** 31 - 1, 0, 1, 2, 3],
              [0, T, 50, 60, 55, T]):
        offsets = torch.tensor(o, dtype=torch.int32, device="cuda")
        a = ntc.linear4(cut(x, B, 0), packed, scales, group=32, rows=rows, offsets=offsets)
        b = ntc.linear4(cut(x, B, 3), shift(packed, 255), shift(scales, math.nan), group=32, rows=rows, offsets=offsets)
        first = min(max(0, min(v, T)) for v in o)  # rows before the first offset have no result
        assert torch.equal(a[first:], b[first:]), o


def test_copied_operands_in_graphs_and_on_streams(ntc):
    packed, scales, _, g = whole(3, 70, 101, 32, H, 5)
    x = [torch.randn(500, 101, generator=g, device="cuda").to(H) for _ in range(3)]
    offsets = torch.tensor([0, 100, 100, 480], dtype=torch.int32, device="cuda")
    want = [ntc.linear4(cut(t, H, 1), packed, scales, group=32, offsets=offsets) for t in x]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    live = [cut(x[0], H, 1), cut(x[0], H, 5)]
    y = ntc.linear4(live[0], packed, scales, group=32, offsets=offsets, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for t, graph in zip(live, graphs):
        with torch.cuda.graph(graph):
            outs.append(ntc.linear4(t, packed, scales, group=32, offsets=offsets))
    for i in (1, 2):
        live[0].copy_(x[i])
        live[1].copy_(x[3 - i])
        torch.cuda.synchronize()
        for graph in graphs:
            with torch.cuda.stream(torch.cuda.Stream()):
                graph.replay()
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[i]) and torch.equal(outs[1], want[3 - i])
