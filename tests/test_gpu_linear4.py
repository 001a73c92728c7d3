"""Weights in 4 bits: packing against its definition, and the product against a 64-bit one."""
import math

import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu
H, B, F = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def randn(*shape, seed=0, std=1.0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("w_type,dtype", [(B, B), (H, H), (F, B), (F, H), (B, H)])
@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (2, 3, 2), (3, 5, 31), (2, 7, 33), (1, 40, 64), (2, 9, 129), (3, 17, 257), (2, 33, 771), (1, 8, 2048)])
def test_pack_and_unpack(ntc, E, N, K, group, w_type, dtype):
    w = randn(E, N, K, seed=K, std=0.3).to(w_type)
    w[..., ::3] *= 0.1
    packed, scales = ntc.pack4(w, group=group, dtype=dtype)
    q, s = S.pack4(w, group, dtype)
    assert packed.dtype == torch.uint8 and packed.shape == (E, N, (K + 1) // 2) and scales.dtype == dtype
    assert torch.equal(scales, s)
    # the reference rounds w / s from 64 bits, half to even: no code may differ
    assert torch.equal(S.nibbles(packed, K), q)
    if K % 2:
        assert bool((packed[..., -1] >> 4 == 8).all())
    back = ntc.unpack4(packed, scales, K, group=group)
    assert torch.equal(back, S.values(packed, scales, K, group).to(dtype)) and back.dtype == dtype
    if E == 1:
        p2, s2 = ntc.pack4(w[0], group=group, dtype=dtype)
        assert torch.equal(p2, packed[0]) and torch.equal(s2, scales[0])
        assert torch.equal(ntc.unpack4(p2, s2, K, group=group), back[0])


def test_halves_go_to_the_even_number(ntc):
    """w / s exactly between two numbers: groups whose largest is 7 have the scale 1."""
    w = torch.arange(-14, 15, device="cuda").to(B)[None] / 2
    w = torch.cat([w, torch.full((1, 3), 7.0, dtype=B, device="cuda")], 1)
    packed, scales = ntc.pack4(w, group=32)
    assert float(scales) == 1.0 and torch.equal(S.nibbles(packed, 32), torch.round(w.double()))


@pytest.mark.parametrize("dtype", [H, B])
def test_groups_that_are_zero_tiny_huge_or_not_numbers(ntc, dtype):
    tiny = 6e-8 if dtype == H else 1e-39
    w = randn(1, 6, 64, seed=4)
    w[0, 0] = 0.0
    w[0, 1, :32] *= tiny
    w[0, 2, 40] = math.nan
    w[0, 3, 3] = math.inf
    w[0, 4] *= 1e4 if dtype == H else 1e38
    w[0, 5, :32] *= tiny * 1e-4
    packed, scales = ntc.pack4(w, group=32, dtype=dtype)
    q, s = S.pack4(w, 32, dtype)
    assert torch.equal(torch.isnan(scales), torch.isnan(s)) and torch.equal(scales[~torch.isnan(s)], s[~torch.isnan(s)])
    assert bool(torch.isnan(scales[0, 2, 1])) and bool(torch.isnan(scales[0, 3, 0])) and not scales[0, 0].any()
    good = ~torch.isnan(s).repeat_interleave(32, -1)
    assert torch.equal(S.nibbles(packed, 64)[good], q[good])
    back = ntc.unpack4(packed, scales, 64, group=32)
    assert bool(torch.isnan(back[~good]).all()) and torch.equal(back[good], S.values(packed, scales, 64, 32).to(dtype)[good])


def test_strided_weights(ntc):
    big = randn(4, 40, 300, seed=8).to(B)
    for w in (big[1:3, 3:20, 1:262], big[::2, ::3, :128], big[3, 5:, 7:201]):
        packed, scales = ntc.pack4(w, group=64)
        p, s = ntc.pack4(w.contiguous(), group=64)
        assert torch.equal(packed, p) and torch.equal(scales, s)
        wide = torch.full(packed.shape[:-1] + (packed.shape[-1] + 9,), 255, dtype=torch.uint8, device="cuda")
        inner = wide[..., 5:5 + packed.shape[-1]]
        inner.copy_(packed)
        padded = torch.full(scales.shape[:-1] + (scales.shape[-1] + 3,), math.nan, dtype=B, device="cuda")[..., 2:2 + scales.shape[-1]]
        padded.copy_(scales)
        assert torch.equal(ntc.unpack4(inner, padded, w.shape[-1], group=64), ntc.unpack4(packed, scales, w.shape[-1], group=64))


def product(ntc, T, E, k, N, K, group, dtype, act="none", bias=True, residual=False, seed=0, odd=False, empty=True):
    g = torch.Generator(device="cuda").manual_seed(seed + T + N + K)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = r(E, N, K) * K ** -0.5
    packed, scales = ntc.pack4(w, group=group, dtype=dtype)
    x = r(T, K + (3 if odd else 0))[:, 1 if odd else 0:][:, :K].to(dtype) if not odd else r(T, K + 3).to(dtype)[:, 1:K + 1]
    rows = offsets = None
    n = T
    if E > 1:
        ids = torch.rand(T, E, generator=g, device="cuda").topk(k, 1).indices.int()
        if empty:
            ids[torch.rand(T, k, generator=g, device="cuda") < 0.2] = -1
            ids[ids == 1] = -1
        rows, _, offsets = R.order(ids, E)
        n = T * k
    b = r(E, N) if bias else None
    res = r(n, N).to(dtype) if residual else None
    if odd:  # packed rows and scales at any address
        p = torch.full((E, N, packed.shape[-1] + 3), 170, dtype=torch.uint8, device="cuda")[..., 1:1 + packed.shape[-1]]
        p.copy_(packed)
        packed = p
        s = torch.full((E, N, scales.shape[-1] + 1), math.nan, dtype=dtype, device="cuda")[..., 1:]
        s.copy_(scales)
        scales = s
    y = ntc.linear4(x, packed, scales, b, group=group, rows=rows, offsets=offsets, activation=act, residual=res)
    values = S.values(packed, scales, K, group)
    want, _, bound, _ = R.linear(x, values, b, rows, offsets, act, residual=res)
    # where the weights are unpacked first they are rounded to 16 bits
    xs = R.gathered(x, rows).abs()
    for e, a, o in R.segments(offsets, n):
        bound[a:o] += 1.2 * R.UNIT[dtype] * (xs[a:o] @ values[e].abs().t()) + R.TINY[dtype] * K
    return y, want, bound


FEW = [(1, 1, 1, 1, 1), (1, 1, 1, 16, 32), (3, 1, 1, 17, 33), (8, 1, 1, 40, 130), (9, 1, 1, 33, 500), (16, 1, 1, 100, 257), (17, 1, 1, 31, 640),
       (31, 1, 1, 257, 96), (32, 1, 1, 128, 2049), (1, 8, 3, 48, 300), (5, 16, 4, 129, 64), (64, 32, 4, 70, 200), (40, 4, 3, 64, 771),
       (1, 64, 8, 200, 1024), (12, 3, 1, 2000, 40)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("T,E,k,N,K", FEW)
def test_few_rows(ntc, T, E, k, N, K, group, dtype):
    y, want, bound = product(ntc, T, E, k, N, K, group, dtype, act="leaky", residual=True)
    R.assert_within(y, want, bound)
    y, want, bound = product(ntc, T, E, k, N, K, group, dtype, odd=True, seed=1)
    R.assert_within(y, want, bound)


@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("T,E,k,N,K", [(33, 1, 1, 40, 64), (200, 1, 1, 65, 771), (500, 4, 2, 128, 256), (300, 3, 2, 33, 129), (2000, 8, 2, 64, 96), (129, 1, 1, 512, 2000)])
def test_many_rows(ntc, T, E, k, N, K, dtype):
    y, want, bound = product(ntc, T, E, k, N, K, 64, dtype, act="silu", residual=True)
    R.assert_within(y, want, bound)
    y, want, bound = product(ntc, T, E, k, N, K, 32, dtype, bias=False, odd=True)
    R.assert_within(y, want, bound)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [B, H])
@pytest.mark.parametrize("T,E,k,N,K", [(40, 1, 1, 8192, 64), (33, 1, 1, 8065, 32), (64, 1, 1, 8300, 96), (100, 1, 1, 8129, 640),
                                       (128, 1, 1, 8200, 2048), (17, 1, 1, 20000, 160), (300, 24, 2, 400, 160), (150, 16, 2, 520, 512),
                                       (96, 16, 2, 600, 224), (1500, 33, 2, 257, 128), (700, 256, 8, 129, 96), (3000, 64, 1, 130, 1056),
                                       (900, 64, 3, 330, 160), (11000, 1024, 1, 130, 64), (129, 1, 1, 8192, 64), (192, 1, 1, 8200, 224), (2000, 32, 2, 260, 352), (193, 1, 1, 8192, 64), (900, 2, 1, 128, 1056), (300, 4, 2, 200, 160)])
def test_rows_in_between(ntc, T, E, k, N, K, group, dtype):
    """Rows of whole 32s that start on 16 bytes: tiles of 32, 64, 128 and 192 rows, experts of several, and, at the end, what
    unpacking and the product for few rows take."""
    y, want, bound = product(ntc, T, E, k, N, K, group, dtype, act="gelu", residual=True)
    R.assert_within(y, want, bound)
    y, want, bound = product(ntc, T, E, k, N, K, group, dtype, bias=False, seed=2, empty=False)
    R.assert_within(y, want, bound)


@pytest.mark.parametrize("T", [300, 900, 2500, 5000])
def test_every_row_to_one_expert(ntc, T):
    """The kernels are chosen for experts of as many rows; one that has them all is right too, and so are no rows at all."""
    E, N, K = 32, 300, 128
    packed, scales = ntc.pack4(randn(E, N, K, seed=T), group=32, dtype=B)
    values = S.values(packed, scales, K, 32)
    x = randn(T, K, seed=T + 1).to(B)
    for e, live in ((0, T), (17, T), (E - 1, T - 5), (3, 0)):
        offsets = torch.tensor([0] * (e + 1) + [live] * (E - e), dtype=torch.int32, device="cuda")
        rows = torch.arange(T, dtype=torch.int32, device="cuda").flip(0).contiguous()
        y = ntc.linear4(x, packed, scales, group=32, rows=rows, offsets=offsets)
        want, _, bound, _ = R.linear(x, values, None, rows, offsets)
        bound[:live] += 1.2 * R.UNIT[B] * (R.gathered(x, rows).abs()[:live] @ values[e].abs().t()) + R.TINY[B] * K
        R.assert_within(y, want, bound)
        assert not y[live:].any()


@pytest.mark.parametrize("act", ["none", "relu", "leaky", "gelu", "silu"])
@pytest.mark.parametrize("T", [4, 100])
def test_activations(ntc, act, T):
    y, want, bound = product(ntc, T, 1, 1, 96, 200, 32, H, act=act)
    R.assert_within(y, want, bound, act)


def test_groups_are_exact_where_the_numbers_are(ntc):
    """Whole numbers whose sums fp32 holds: few rows give the exact product, whatever the scales' rounding would do to a
    weight (scales of 11 bits times q have up to 15)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    K, N = 512, 48
    q = torch.randint(-8, 8, (N, K), generator=g, device="cuda")
    s = (torch.randint(1, 2048, (N, K // 32), generator=g, device="cuda").double() / 64).to(H)
    x = torch.randint(-3, 4, (7, K), generator=g, device="cuda").to(H)
    packed = ((q[:, 0::2] + 8) | (q[:, 1::2] + 8) << 4).to(torch.uint8)
    y = ntc.linear4(x, packed, s, group=32)
    want = (x.double() @ (q.double() * s.double().repeat_interleave(32, -1)).t())
    assert torch.equal(y, want.to(H))


@pytest.mark.parametrize("T", [6, 400])
def test_offsets_that_are_anything(ntc, T):
    """Offsets outside the rows or decreasing, rows outside x: results stay inside their buffers, and experts share no row."""
    E, N, K = 5, 40, 96
    packed, scales = ntc.pack4(randn(E, N, K, seed=2).to(B), group=32)
    w = ntc.unpack4(packed, scales, K, group=32)
    x = randn(T, K, seed=3).to(B)
    rows = torch.arange(T, dtype=torch.int32, device="cuda")
    rows[::5] = -1
    rows[1::5] = 2 ** 31 - 1
    for o in ([0, 0, 2, 1, 4, T], [-5, 3, 3, 3, 4, 10 * T], [T] * 6, [0] * 6, [2, 1, 0, 3, 2, T // 2], [-2 ** 31, 2 ** 31 - 1, 0, 1, 2, 3]):
        offsets = torch.tensor(o, dtype=torch.int32, device="cuda")
        y = ntc.linear4(x, packed, scales, group=32, rows=rows, offsets=offsets)
        z = ntc.linear(x, w, rows=rows, offsets=offsets)
        least = torch.tensor([min(max(0, min(v, T)) for v in o[e:]) for e in range(E + 1)])
        for e in range(E):
            a, b = int(least[e]), int(least[e + 1])
            want = R.gathered(x, rows[a:b]) @ w[e].double().t()
            mag = R.gathered(x, rows[a:b]).abs() @ w[e].double().abs().t()
            for got in (y[a:b], z[a:b]):
                R.assert_within(got, want, mag * (2 * 2.0 ** -8) + 1e-30, (o, e))
        assert not y[int(least[E]):].any()


def test_padding_and_neighbours_are_not_read(ntc):
    """NaN around x, 255 around packed, NaN around the scales; rows of no expert hold NaN in the residual."""
    for T in (3, 20, 90):
        K, N, E = 200, 33, 3
        packed, scales = ntc.pack4(randn(E, N, K, seed=T).to(H), group=64)
        x = torch.full((T + 2, K + 16), math.nan, dtype=H, device="cuda")
        x[1:-1, 8:8 + K] = randn(T, K, seed=T + 1).to(H)
        x = x[1:-1, 8:8 + K]
        p = torch.full((E, N + 1, packed.shape[-1] + 16), 255, dtype=torch.uint8, device="cuda")
        p[:, :N, 16:] = packed
        s = torch.full((E, N + 1, scales.shape[-1] + 4), math.nan, dtype=H, device="cuda")
        s[:, :N, 2:-2] = scales
        offsets = torch.tensor([0, T // 3, T // 3, T - 1], dtype=torch.int32, device="cuda")
        res = randn(T, N, seed=9).to(H)
        res[T - 1] = math.nan
        a = ntc.linear4(x, p[:, :N, 16:], s[:, :N, 2:-2], group=64, offsets=offsets, residual=res)
        b = ntc.linear4(x.contiguous(), packed, scales, group=64, offsets=offsets, residual=res)
        assert torch.equal(a, b) and bool(torch.isfinite(a).all()) and not a[T - 1].any()


def test_streams_graphs_and_equal_bits(ntc):
    for T in (5, 30, 300):
        packed, scales = ntc.pack4(randn(4, 64, 256, seed=1).to(B), group=64)
        x = randn(T, 256, seed=2).to(B)
        offsets = torch.tensor([0, T // 4, T // 2, T // 2, T], dtype=torch.int32, device="cuda")
        call = lambda **k: ntc.linear4(x, packed, scales, group=64, offsets=offsets, **k)  # noqa: E731
        y = call()
        assert torch.equal(y, call())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        z = call(stream=side)
        side.synchronize()
        assert torch.equal(y, z)
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        outs = []
        for g in graphs:
            with torch.cuda.graph(g):
                outs.append(call())
        x.copy_(randn(T, 256, seed=3).to(B))
        offsets.copy_(torch.tensor([0, 1, 2, T // 2, T], dtype=torch.int32))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = call()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("T,N", [(500, 33), (700, 150), (3000, 120), (9000, 60)])
def test_tiles_in_between_read_nothing_else_and_repeat(ntc, T, N):
    """64 experts: NaN and 255 around the operands, on both sides of a padded batch; two graphs at once on two streams."""
    E, K = 64, 224
    packed, scales = ntc.pack4(randn(E, N, K, seed=T).to(B), group=64)
    x = torch.full((T + 2, K + 16), math.nan, dtype=B, device="cuda")
    x[1:-1, 8:8 + K] = randn(T, K, seed=T + 1).to(B)
    x = x[1:-1, 8:8 + K]
    p = torch.full((E, N + 1, 112 + 32), 255, dtype=torch.uint8, device="cuda")
    p[:, :N, 16:128] = packed
    p = p[:, :N, 16:128]
    s = torch.full((E, N + 1, scales.shape[-1] + 3), math.nan, dtype=B, device="cuda")
    s[:, :N, 1:-2] = scales
    s = s[:, :N, 1:-2]
    res = torch.full((T, N + 5), math.nan, dtype=B, device="cuda")
    res[:T - 9, 2:2 + N] = randn(T - 9, N, seed=9).to(B)
    cuts = torch.sort(torch.randint(0, T - 8, (E + 1,), generator=torch.Generator(device="cuda").manual_seed(N), device="cuda"))[0].int()
    cuts[0], cuts[-1] = 0, T - 9
    call = lambda: ntc.linear4(x, p, s, group=64, offsets=cuts, residual=res[:, 2:2 + N], activation="silu")  # noqa: E731
    y = call()
    assert torch.equal(y, ntc.linear4(x.contiguous(), packed, scales, group=64, offsets=cuts, residual=res[:, 2:2 + N].contiguous(), activation="silu"))
    assert bool(torch.isfinite(y).all()) and not y[T - 9:].any()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(call())
    x.copy_(randn(T, K, seed=3).to(B))
    cuts[1:9] = cuts[9].clone()
    torch.cuda.synchronize()
    for g in graphs:
        with torch.cuda.stream(torch.cuda.Stream()):
            g.replay()
            g.replay()
    torch.cuda.synchronize()
    want = call()
    assert not torch.equal(want, y) and torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_no_rows(ntc):
    packed, scales = ntc.pack4(randn(2, 8, 64).to(B), group=32)
    y = ntc.linear4(torch.zeros(0, 64, dtype=B, device="cuda"), packed, scales, group=32, offsets=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert y.shape == (0, 8)


@pytest.mark.parametrize("T", [2, 40])
def test_weights_past_2_31_bytes(ntc, T):
    """Three experts of 65,536 x 28,672 weights: 2.8 GB packed, offsets past 32 bits in bytes and in weights."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    E, N, K = 3, 65536, 28672
    packed = torch.randint(0, 256, (E, N, K // 2), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    scales = torch.full((E, N, K // 128), 2.0 ** -8, dtype=B, device="cuda")
    x = randn(T, K, seed=5).to(B)
    offsets = torch.tensor([0, 1, 1, T], dtype=torch.int32, device="cuda")
    y = ntc.linear4(x, packed, scales, group=128, offsets=offsets)
    some = torch.tensor([0, 1, 4097, 65535], device="cuda")
    for e, a, b in ((0, 0, 1), (2, 1, T)):
        w = S.values(packed[e][some], scales[e][some], K, 128)
        want, mag = x[a:b].double() @ w.t(), x[a:b].double().abs() @ w.abs().t()
        R.assert_within(y[a:b][:, some], want, mag * (K + 8) * R.F32 + want.abs() * 2.0 ** -7 + 1e-30, e)


def test_what_is_refused(ntc):
    z = lambda *s, dtype=H: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    U = torch.uint8
    for call, word in [
            (lambda: ntc.pack4(z(8)), "two or three"), (lambda: ntc.pack4(z(8, 4).t()), "last dimension"), (lambda: ntc.pack4(z(4, 8), group=48), "group"),
            (lambda: ntc.pack4(z(4, 8), dtype=F), "dtype"), (lambda: ntc.pack4(z(4, 8, dtype=torch.float64)), "float32, float16"),
            (lambda: ntc.pack4(torch.zeros(4, 8)), "CUDA tensor"), (lambda: ntc.pack4(z(0, 8)), "shape"),
            (lambda: ntc.unpack4(z(4, 5, dtype=U), z(4, 1), 8), "shape"), (lambda: ntc.unpack4(z(4, 4, dtype=U), z(4, 2), 8), "shape"),
            (lambda: ntc.unpack4(z(4, 4), z(4, 1), 8), "must be Byte"), (lambda: ntc.unpack4(z(4, 4, dtype=U), z(4, 1), -1), "d_in"),
            (lambda: ntc.linear4(z(2, 8), z(4, 4, dtype=U), z(4, 1, dtype=B)), "scales must be Half"),
            (lambda: ntc.linear4(z(2, 9), z(4, 4, dtype=U), z(4, 1)), "shape"), (lambda: ntc.linear4(z(2, 8), z(4, 4, dtype=U), z(4, 1), z(5, dtype=F)), "shape"),
            (lambda: ntc.linear4(z(2, 8), z(4, 4, dtype=U), z(4, 1), residual=z(2, 5)), "shape"),
            (lambda: ntc.linear4(z(2, 8), z(4, 4, dtype=U), z(4, 1), activation="tanh"), "activation")]:
        with pytest.raises(ValueError, match=word):
            call()
    with pytest.raises(TypeError):
        ntc.pack4(z(4, 8), dtype="fp16")
    for call, word in [(lambda: ntc.unpack4(z(4, 4, dtype=U), z(4, 1, dtype=F), 8), "fp16 or bf16"),
                       (lambda: ntc.linear4(z(2, 8), z(2, 4, 4, dtype=U), z(2, 4, 1)), "offsets"),
                       (lambda: ntc.linear4(z(2, 8), z(4, 4, dtype=U), z(4, 1), leaky_slope=math.nan), "leaky_slope")]:
        with pytest.raises(ntc.NtcError, match=word):
            call()
