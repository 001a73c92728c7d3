"""The linear layers with offsets that are not what they ask for: an offset outside 0..rows counts as the nearer
end, one above a later offset as that one, and nothing outside the buffers and the workspace's stated size is written."""
import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu
GUARD = 4096


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    yield ntc
    ntc.ntc_linear_status(0)


def held(offsets, n):
    least, out = n, []
    for o in reversed(offsets):
        least = min(least, max(0, min(n, o)))
        out.insert(0, least)
    return out


class Guarded:
    """A buffer with 4 KB of a known byte on both sides."""

    def __init__(self, size):
        self.all = torch.full((size + 2 * GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
        self.size, self.ptr = size, self.all.data_ptr() + GUARD

    def view(self, dtype, *shape):
        return self.all[GUARD:GUARD + self.size].view(dtype).view(*shape)

    def whole(self):
        return bool((self.all[:GUARD] == 0x5A).all()) and bool((self.all[GUARD + self.size:] == 0x5A).all())


WILD = {"twice the rows": lambda E, n: [0 if e % 2 == 0 else n for e in range(E + 1)],
        "falling": lambda E, n: [n - e * (n // (E + 1)) for e in range(E + 1)],
        "outside": lambda E, n: [-7] + [n // 3] * (E - 1) + [2 ** 31 - 1],
        "a dip": lambda E, n: [0] + [n // 2 if e != E // 2 else n // 4 for e in range(1, E)] + [n]}


@pytest.mark.parametrize("what", WILD)
@pytest.mark.parametrize("n,E,K,N", [(1280, 3, 64, 64), (12, 3, 64, 64), (1000, 33, 72, 136), (3000, 2, 1096, 4104)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_wild_offsets(ntc, what, n, E, K, N, act):
    g = torch.Generator(device="cuda").manual_seed(n + E)
    offsets = WILD[what](E, n)
    want = held(offsets, n)
    good = torch.tensor(want, dtype=torch.int32)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()
    x, w, dy, z = normal(n, K), normal(E, N, K, std=K ** -0.5), normal(n, N), normal(n, N)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    d = ntc.ntc_linear_desc(ntc.NTC_TYPE_BF16, K, N, E, ntc.ACTIVATIONS[act], 0.0, n, n, K, K, N * K, N, N, N)
    stream = torch.cuda.current_stream().cuda_stream
    live = slice(want[0], n)

    y = Guarded(n * N * 2)
    ws = Guarded(ntc.ntc_linear_workspace(d, x.data_ptr(), None, w.data_ptr()))
    ntc.ntc_linear(d, x.data_ptr(), None, off.data_ptr(), w.data_ptr(), None, None, y.ptr, None, ws.ptr, ws.size, stream)
    ref, _, bound, _ = R.linear(x, w, None, None, good, act)
    R.assert_within(y.view(torch.bfloat16, n, N)[live], ref[live], bound[live], "y")
    assert y.whole() and ws.whole()

    refs = R.linear_backward(dy, x, w, z, None, good, act)
    for need in (("dx", "dw", "db"), ("db",), ("dx", "db")):
        out = {"dx": Guarded(n * K * 2), "dw": Guarded(E * N * K * 2), "db": Guarded(E * N * 4)}
        ptr = [out[k].ptr if k in need else None for k in ("dx", "dw", "db")]
        ws = Guarded(ntc.ntc_linear_backward_workspace(d, dy.data_ptr(), x.data_ptr(), None, w.data_ptr()))
        ntc.ntc_linear_backward(d, dy.data_ptr(), z.data_ptr(), x.data_ptr(), None, off.data_ptr(), w.data_ptr(), *ptr, ws.ptr,
                                ws.size, stream)
        got = {"dx": out["dx"].view(torch.bfloat16, n, K)[live], "dw": out["dw"].view(torch.bfloat16, E, N, K),
               "db": out["db"].view(torch.float32, E, N)}
        for k, (ref, bound) in zip(("dx", "dw", "db"), refs):
            if k in need:
                R.assert_within(got[k], ref[live] if k == "dx" else ref, bound[live] if k == "dx" else bound, k)
            assert out[k].whole()
        assert ws.whole()
