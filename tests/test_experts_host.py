"""Refusals of the routed-expert calls: every one of them before any device work."""
import ctypes

import pytest

from paper_2608_27888_gb300 import build as B

B.build()
from paper_2608_27888_gb300 import ntc  # noqa: E402

BAD, UNSUPPORTED = ntc.NTC_ERR_INVALID_ARG, ntc.NTC_ERR_UNSUPPORTED
P = 1 << 20  # an address that is never followed


def made(cls, defaults, over):
    d = cls()
    for k, v in {**defaults, **over}.items():
        setattr(d, k, v)
    return ctypes.byref(d)


ROUTE = dict(num_experts=64, top_k=4, num_groups=8, top_groups=2, score=0, renormalize=1, scale=1.0, type=0)
LINEAR = dict(type=2, in_dim=64, out_dim=32, num_experts=4, activation=1, leaky_slope=0.0, num_rows=10, num_x_rows=5, ld_x=64,
              ld_w=64, stride_w=2048, ld_y=32, ld_z=32, ld_residual=32)
COMBINE = dict(type=2, dim=32, top_k=2, num_experts=4, num_tokens=5, num_rows=10, ld_y=32, ld_out=32, ld_residual=32)


def test_descriptor_layouts_match_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for cls in (ntc.ntc_route_desc, ntc.ntc_linear_desc, ntc.ntc_combine_desc):
        name, fields = cls.__name__, [f for f, _ in cls._fields_]
        src = tmp_path / f"{name}.c"
        body = "\n".join(f'  printf("%zu\\n", offsetof({name}, {f}));' for f in fields)
        src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"ntc.h\"\nint main(void) {\n" + body +
                       f'\n  printf("%zu\\n", sizeof({name}));\n  return 0;\n}}\n')
        exe = tmp_path / name
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
        got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
        assert got == [getattr(cls, f).offset for f in fields] + [ctypes.sizeof(cls)]


@pytest.mark.parametrize("over,word", [
    (dict(num_experts=0), "num_experts"), (dict(num_experts=1025), "num_experts"), (dict(top_k=0), "top_k"),
    (dict(top_k=33), "top_k"), (dict(num_experts=8, num_groups=1, top_groups=1, top_k=9), "top_k"), (dict(num_groups=7), "num_groups"), (dict(num_groups=64), "num_groups"),
    (dict(num_groups=0), "num_groups"), (dict(top_groups=0), "top_groups"), (dict(top_groups=9), "top_groups"),
    (dict(top_groups=1, top_k=9), "top_k"), (dict(score=2), "score"), (dict(renormalize=2), "renormalize"),
    (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(type=3), "type")])
def test_route_refusals(over, word):
    d = made(ntc.ntc_route_desc, ROUTE, over)
    assert ntc._lib.ntc_route(d, 4, P, 1024, None, P, P, None) == BAD
    assert word in ntc.ntc_last_error()


def test_route_pointer_refusals():
    d = made(ntc.ntc_route_desc, ROUTE, {})
    r, back = ntc._lib.ntc_route, ntc._lib.ntc_route_backward
    assert r(None, 4, P, 64, None, P, P, None) == BAD
    assert r(d, 4, None, 64, None, P, P, None) == BAD
    assert r(d, 4, P, 64, None, None, P, None) == BAD
    assert r(d, 4, P, 64, None, P, None, None) == BAD
    assert r(d, 4, P, 63, None, P, P, None) == BAD
    assert r(d, 1 << 31, P, 64, None, P, P, None) == BAD
    assert r(d, 4, P + 2, 64, None, P, P, None) == BAD
    assert r(d, 4, P, 64, P + 1, P, P, None) == BAD
    assert r(d, 0, None, 64, None, None, None, None) == ntc.NTC_OK
    assert back(d, 4, P, 64, P, None, P, None) == BAD
    assert back(d, 4, P, 64, P, P, P + 1, None) == BAD
    assert back(d, 0, None, 64, None, None, None, None) == ntc.NTC_OK


def test_order_refusals():
    f, ws = ntc._lib.ntc_expert_order, ntc._lib.ntc_expert_order_workspace
    assert ws(100, 64) == 0 and ws(1 << 20, 64) > 0 and ws(1 << 31, 64) == 0 and ws(100000, 0) == 0
    n = 100000
    assert f(P, n, 8, 0, P, P, P, P, 1 << 30, None) == BAD
    assert f(P, n, 8, 1025, P, P, P, P, 1 << 30, None) == BAD
    assert f(P, n, 0, 64, P, P, P, P, 1 << 30, None) == BAD
    assert f(P, n, 33, 64, P, P, P, P, 1 << 30, None) == BAD
    assert f(P, n, 3, 64, P, P, P, P, 1 << 30, None) == BAD  # not a multiple
    assert f(None, n, 8, 64, P, P, P, P, 1 << 30, None) == BAD
    assert f(P, n, 8, 64, P, P, None, P, 1 << 30, None) == BAD
    assert f(P, n, 8, 64, P, P, P, P, ws(n, 64) - 1, None) == BAD
    assert f(P, n, 8, 64, P, P, P, None, 1 << 30, None) == BAD
    assert f(P, n, 8, 64, P, P, P, P + 4, 1 << 30, None) == BAD
    assert f(P + 2, n, 8, 64, P, P, P, P, 1 << 30, None) == BAD


@pytest.mark.parametrize("over,status,word", [
    (dict(type=0), UNSUPPORTED, "fp16 or bf16"), (dict(type=5), BAD, "type"), (dict(in_dim=0), BAD, "in_dim"),
    (dict(in_dim=(1 << 20) + 1), BAD, "in_dim"), (dict(out_dim=0), BAD, "out_dim"), (dict(num_experts=0), BAD, "num_experts"),
    (dict(num_experts=1025), BAD, "num_experts"), (dict(activation=5), BAD, "activation"),
    (dict(leaky_slope=float("nan")), BAD, "leaky_slope"), (dict(num_rows=1 << 31), BAD, "rows"), (dict(ld_x=63), BAD, "ld_x"),
    (dict(ld_w=63), BAD, "ld_w"), (dict(ld_y=31), BAD, "ld_y"), (dict(ld_z=31), BAD, "ld_z"),
    (dict(ld_residual=31), BAD, "ld_residual"), (dict(ld_y=1 << 39), UNSUPPORTED, "2^38"), (dict(stride_w=2047), BAD, "stride_w"),
    (dict(num_x_rows=0), BAD, "no rows")])
def test_linear_refusals(over, status, word):
    d = made(ntc.ntc_linear_desc, LINEAR, over)
    assert ntc._lib.ntc_linear(d, P, P, P, P, P, P, P, P, P, 1 << 40, None) == status
    assert word in ntc.ntc_last_error()
    assert ntc._lib.ntc_linear_backward(d, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == status


def test_linear_pointer_refusals():
    d = made(ntc.ntc_linear_desc, LINEAR, {})
    f, b = ntc._lib.ntc_linear, ntc._lib.ntc_linear_backward
    good = [P, P, P, P, None, None, P, None, None, 0]

    def call(fn, base, i, v):
        a = list(base)
        a[i] = v
        return fn(d, *a, None)
    for i in (0, 3, 6):
        assert call(f, good, i, None) == BAD
    for i in (0, 3, 4, 5, 6, 7):
        assert call(f, good, i, P + 1) == BAD
    assert call(f, good, 1, None) == BAD  # no rows, and num_x_rows differs
    assert call(f, good, 2, None) == BAD  # several experts without offsets
    assert call(f, good, 1, P + 2) == BAD
    odd = made(ntc.ntc_linear_desc, LINEAR, dict(ld_x=65, num_rows=1000))
    even = made(ntc.ntc_linear_desc, LINEAR, dict(num_rows=1000))
    need = ntc._lib.ntc_linear_workspace(odd, P, P, P)
    assert need > 0 and ntc._lib.ntc_linear_workspace(even, P, P, P) == 0
    assert ntc._lib.ntc_linear_workspace(even, P + 8, P, P) > 0 and ntc._lib.ntc_linear_workspace(even, P, P, P + 2) > 0
    assert ntc._lib.ntc_linear_workspace(d, P + 8, P, P + 2) == 0  # few rows are read where they lie
    big = made(ntc.ntc_linear_desc, LINEAR, dict(num_rows=65536, in_dim=2048, ld_x=2048, ld_w=2048, out_dim=4096, ld_y=4096,
                                                 ld_z=4096, ld_residual=4096, stride_w=2048 * 4096))
    assert ntc._lib.ntc_linear_workspace(big, P, P, P) >= 65536 * 2048 * 2  # gathered rows in order
    assert ntc._lib.ntc_linear_workspace(big, P, None, P) == 0
    assert f(odd, *good[:8], P, need - 1, None) == BAD
    assert f(odd, *good[:8], None, need, None) == BAD
    assert f(odd, *good[:8], P + 8, need, None) == BAD
    assert f(None, *good, None) == BAD
    need = ntc._lib.ntc_linear_backward_workspace(d, P, P, P, P)
    back = [P, P, P, P, P, P, P, P, P, P, need]
    for i in (0, 1, 2, 5):  # dy, z, x, w
        assert call(b, back, i, None) == BAD
    for i in (0, 1, 2, 5, 6, 7, 8):
        assert call(b, back, i, P + 1) == BAD
    assert call(b, back, 10, need - 1) == BAD
    assert b(d, P, P, P, P, P, P, None, None, None, P, need, None) == ntc.NTC_OK  # nothing asked for
    refused = made(ntc.ntc_linear_desc, LINEAR, dict(in_dim=0))
    assert ntc._lib.ntc_linear_workspace(refused, P, P, P) == 0
    assert ntc._lib.ntc_linear_backward_workspace(refused, P, P, P, P) == 0


@pytest.mark.parametrize("over", [dict(type=4), dict(dim=0), dict(dim=(1 << 20) + 1), dict(top_k=0), dict(top_k=33),
                                  dict(num_experts=0), dict(num_experts=2000), dict(num_rows=1 << 31), dict(num_tokens=1 << 31),
                                  dict(ld_y=31), dict(ld_out=31), dict(ld_residual=31)])
def test_combine_refusals(over):
    d = made(ntc.ntc_combine_desc, COMBINE, over)
    assert ntc._lib.ntc_combine(d, P, P, P, P, P, P, None) == BAD
    assert ntc._lib.ntc_combine_backward(d, P, P, P, P, P, P, P, None) == BAD


def test_combine_pointer_refusals():
    d = made(ntc.ntc_combine_desc, COMBINE, {})
    f, b = ntc._lib.ntc_combine, ntc._lib.ntc_combine_backward
    for a in ((None, P, P, P, P, P), (P, None, P, P, P, P), (P, P, P, P, P, None), (P + 1, P, P, P, P, P), (P, P + 2, P, P, P, P),
              (P, P, P + 1, P, P, P), (P, P, P, P + 1, P, P), (P, P, P, P, P + 1, P), (P, P, P, P, P, P + 1)):
        assert f(d, *a, None) == BAD
    for a in ((None, P, P, P, P, P, P), (P, None, P, P, P, P, P), (P, P, None, P, P, P, P), (P + 1, P, P, P, P, P, P),
              (P, P, P, P, P, P + 1, P), (P, P, P, P, P, P, P + 2)):
        assert b(d, *a, None) == BAD
    assert b(d, P, P, P, P, P, None, None, None) == ntc.NTC_OK
    none = made(ntc.ntc_combine_desc, COMBINE, dict(num_tokens=0))
    assert f(none, None, None, None, None, None, None, None) == ntc.NTC_OK


def test_the_python_functions_check_their_arguments():
    import torch
    cpu = torch.zeros(2, 8)
    ids = torch.zeros(2, 1, dtype=torch.int32)
    for call in (lambda: ntc.route(cpu, 2), lambda: ntc.route_backward(cpu, ids, cpu[:, :1]), lambda: ntc.linear(cpu, cpu),
                 lambda: ntc.linear_backward(cpu, cpu, cpu), lambda: ntc.combine(cpu, ids),
                 lambda: ntc.combine_backward(cpu, cpu, ids), lambda: ntc.expert_order(ids, 2)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(TypeError, match="w must be a tensor"):
        ntc.linear(cpu, [1.0])
    with pytest.raises(ValueError, match="activation must be one of"):
        ntc.linear(cpu, cpu, activation="tanh")
    with pytest.raises(ValueError, match="score must be one of"):
        ntc.route(cpu, 2, score="max")
    with pytest.raises(ValueError, match="need must name"):
        ntc.linear_backward(cpu, cpu, cpu, need=("dz",))
    with pytest.raises(ValueError, match="need must name"):
        ntc.combine_backward(cpu, cpu, ids, need=("y",))
    with pytest.raises(AttributeError):
        ntc.no_such_name
