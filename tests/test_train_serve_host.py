"""Refusals of the balance loss, the optimizer's step and the 4-bit weights: every one of them before any device work."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_27888_gb300 import build as B

B.build()
from paper_2608_27888_gb300 import ntc  # noqa: E402

BAD, UNSUPPORTED, OK = ntc.NTC_ERR_INVALID_ARG, ntc.NTC_ERR_UNSUPPORTED, ntc.NTC_OK
P = 1 << 20  # an address that is never followed


def made(cls, defaults, over):
    d = cls()
    for k, v in {**defaults, **over}.items():
        setattr(d, k, v)
    return ctypes.byref(d)


BALANCE = dict(num_experts=64, top_k=4, score=0, scale=1.0, type=0)
ADAMW = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0, step=1, moment_bits=32)
PACK = dict(type=2, in_dim=100, out_dim=32, num_experts=4, group=32, ld_packed=64, stride_packed=2048, ld_scales=4, stride_scales=128)
LINEAR = dict(type=2, in_dim=100, out_dim=32, num_experts=4, activation=1, leaky_slope=0.0, num_rows=10, num_x_rows=5, ld_x=104,
              ld_w=0, stride_w=0, ld_y=32, ld_z=0, ld_residual=32)


def test_descriptor_layouts_match_the_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for cls in (ntc.ntc_balance_desc, ntc.ntc_adamw_tensor, ntc.ntc_adamw_desc, ntc.ntc_pack4_desc):
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
    (dict(num_experts=0), "num_experts"), (dict(num_experts=1025), "num_experts"), (dict(top_k=0), "top_k"), (dict(top_k=33), "top_k"),
    (dict(score=2), "score"), (dict(scale=float("nan")), "scale"), (dict(type=3), "type")])
def test_balance_refusals(over, word):
    d = made(ntc.ntc_balance_desc, BALANCE, over)
    assert ntc._lib.ntc_balance_loss(d, 4, P, 1024, P, P, P, P, P, 1 << 30, None) == BAD
    assert word in ntc.ntc_last_error()
    assert ntc._lib.ntc_balance_loss_backward(d, 4, P, 1024, P, P, None, None, 0, P, None) == BAD
    assert ntc._lib.ntc_balance_loss_workspace(d, 1 << 20) == 0


def test_balance_pointer_refusals():
    d = made(ntc.ntc_balance_desc, BALANCE, {})
    f, b, ws = ntc._lib.ntc_balance_loss, ntc._lib.ntc_balance_loss_backward, ntc._lib.ntc_balance_loss_workspace
    n = 100000
    need = ws(d, n)
    assert need > 0 and ws(d, 1) == 0 and ws(d, 1 << 31) == 0
    for bad in range(5):  # logits, ids, loss, counts, mean
        p = [P] * 5
        p[bad] = None
        assert f(d, n, p[0], 64, p[1], p[2], p[3], p[4], P, need, None) == BAD
        p[bad] = P + 2
        assert f(d, n, p[0], 64, p[1], p[2], p[3], p[4], P, need, None) == BAD
    assert f(d, n, P, 63, P, P, P, P, P, need, None) == BAD
    assert f(d, n, P, 64, P, P, P, P, P, need - 1, None) == BAD
    assert f(d, n, P, 64, P, P, P, P, None, need, None) == BAD
    assert f(d, n, P, 64, P, P, P, P, P + 4, need, None) == BAD
    assert f(d, 1 << 29, P, 64, P, P, P, P, P, 1 << 40, None) == BAD  # n * top_k
    for bad in range(4):  # logits, ids, counts, dlogits
        p = [P] * 4
        p[bad] = None
        assert b(d, n, p[0], 64, p[1], p[2], None, None, 0, p[3], None) == BAD
    assert b(d, n, P, 64, P, P, P + 1, None, 0, P, None) == BAD
    assert b(d, n, P, 64, P, P, None, P, 63, P, None) == BAD
    assert b(d, 0, None, 64, None, None, None, None, 0, None, None) == OK


def tensor(**over):
    t = ntc.ntc_adamw_tensor()
    for k, v in {**dict(param=1 << 20, grad=2 << 20, m=3 << 20, v=4 << 20, scale_m=5 << 20, scale_v=6 << 20, copy=7 << 20, count=1000,
                        param_type=0, grad_type=2, copy_type=2), **over}.items():
        setattr(t, k, v)
    return t


def adamw(d, tensors, lr=None, step=None, scale=None, ws=None, size=0):
    t = (ntc.ntc_adamw_tensor * max(1, len(tensors)))(*tensors)
    return ntc._lib.ntc_adamw(d, t, len(tensors), lr, step, scale, ws, size, None)


@pytest.mark.parametrize("over,word", [
    (dict(lr=float("nan")), "finite"), (dict(eps=float("inf")), "finite"), (dict(grad_scale=float("nan")), "finite"),
    (dict(lr=-1.0), "negative"), (dict(eps=-1e-9), "negative"), (dict(weight_decay=-0.1), "negative"), (dict(beta1=1.0), "beta1"),
    (dict(beta2=-0.1), "beta1"), (dict(step=0), "step"), (dict(moment_bits=16), "moment_bits")])
def test_adamw_refusals(over, word):
    assert adamw(made(ntc.ntc_adamw_desc, ADAMW, over), [tensor()]) == BAD
    assert word in ntc.ntc_last_error()


@pytest.mark.parametrize("bits,over,word", [
    (32, dict(param=None), "null"), (32, dict(v=None), "null"), (8, dict(scale_m=None), "null"), (32, dict(param_type=3), "type"),
    (32, dict(copy_type=4), "type"), (32, dict(param=(1 << 20) + 2), "aligned"), (32, dict(m=(3 << 20) + 1), "aligned"),
    (8, dict(scale_v=(6 << 20) + 2), "aligned"), (32, dict(copy=(7 << 20) + 1), "aligned"), (32, dict(count=1 << 40), "2^40"),
    (32, dict(grad=(1 << 20) + 3998), "overlaps"), (32, dict(m=4 << 20), "overlaps"), (32, dict(copy=(4 << 20) - 2), "overlaps"),
    (8, dict(scale_v=(5 << 20) + 12), "overlaps"), (8, dict(m=(1 << 20) + 3999), "overlaps")])
def test_adamw_tensor_refusals(bits, over, word):
    d = made(ntc.ntc_adamw_desc, ADAMW, dict(moment_bits=bits))
    assert adamw(d, [tensor(**over)]) == BAD
    assert word in ntc.ntc_last_error()


def test_adamw_lists():
    d = made(ntc.ntc_adamw_desc, ADAMW, {})
    far = dict(param=1 << 30, m=3 << 30, v=4 << 30, copy=None)
    assert adamw(d, [tensor(), tensor()]) == BAD and "overlaps" in ntc.ntc_last_error()
    assert adamw(d, [tensor(), tensor(param=(1 << 20) + 3996, m=far["m"], v=far["v"], copy=None)]) == BAD
    assert adamw(d, [tensor(), tensor(**far, count=(1 << 39))]) in (BAD, UNSUPPORTED)
    assert adamw(d, []) == OK and adamw(d, [tensor(count=0, param=None)]) == OK
    assert adamw(None, [tensor()]) == BAD
    assert ntc._lib.ntc_adamw(d, None, 1, None, None, None, None, 0, None) == BAD
    assert adamw(d, [tensor()], lr=8 << 20) == BAD and "workspace" in ntc.ntc_last_error()
    assert adamw(d, [tensor()], step=8 << 20, ws=9 << 20, size=15) == BAD
    assert adamw(d, [tensor()], scale=(8 << 20) + 2, ws=9 << 20, size=16) == BAD
    assert adamw(d, [tensor()], scale=8 << 20, ws=(9 << 20) + 8, size=16) == BAD


@pytest.mark.parametrize("over,status,word", [
    (dict(type=0), UNSUPPORTED, "fp16 or bf16"), (dict(type=3), BAD, "type"), (dict(in_dim=0), BAD, "in_dim"),
    (dict(in_dim=(1 << 20) + 1), BAD, "in_dim"), (dict(out_dim=0), BAD, "out_dim"), (dict(num_experts=0), BAD, "num_experts"),
    (dict(num_experts=1025), BAD, "num_experts"), (dict(group=16), BAD, "group"), (dict(group=96), BAD, "group"),
    (dict(ld_packed=49), BAD, "ld_packed"), (dict(ld_scales=3), BAD, "ld_scales"), (dict(stride_packed=31 * 64 + 49), BAD, "stride"),
    (dict(stride_scales=127), BAD, "stride"), (dict(ld_packed=1 << 38, stride_packed=1 << 50), UNSUPPORTED, "2^38")])
def test_pack4_refusals(over, status, word):
    d = made(ntc.ntc_pack4_desc, PACK, over)
    assert ntc._lib.ntc_pack4(d, P, 0, 100, 3200, P, P, None) == status
    assert word in ntc.ntc_last_error()
    assert ntc._lib.ntc_unpack4(d, P, P, P, 100, 3200, None) == status
    l = made(ntc.ntc_linear_desc, LINEAR, {k: v for k, v in over.items() if k in ("in_dim", "out_dim", "num_experts", "type")})
    assert ntc._lib.ntc_linear4(l, d, P, P, P, P, P, P, P, P, P, 1 << 40, None) == status


def test_pack4_pointer_refusals():
    d = made(ntc.ntc_pack4_desc, PACK, {})
    f, b = ntc._lib.ntc_pack4, ntc._lib.ntc_unpack4
    assert f(d, None, 0, 100, 3200, P, P, None) == BAD and f(d, P, 0, 100, 3200, None, P, None) == BAD
    assert f(d, P, 0, 100, 3200, P, None, None) == BAD and f(None, P, 0, 100, 3200, P, P, None) == BAD
    assert f(d, P, 4, 100, 3200, P, P, None) == BAD and f(d, P, 0, 99, 3200, P, P, None) == BAD
    assert f(d, P, 0, 100, 3199, P, P, None) == BAD and f(d, P + 2, 0, 100, 3200, P, P, None) == BAD
    assert f(d, P + 1, 1, 100, 3200, P, P, None) == BAD and f(d, P, 0, 100, 3200, P, P + 1, None) == BAD
    assert f(d, P, 0, 1 << 38, 1 << 50, P, P, None) == UNSUPPORTED
    assert b(d, P, P, None, 100, 3200, None) == BAD and b(d, P, P, P + 1, 100, 3200, None) == BAD


def test_linear4_refusals():
    f, ws = ntc._lib.ntc_linear4, ntc._lib.ntc_linear4_workspace
    l, p = made(ntc.ntc_linear_desc, LINEAR, {}), made(ntc.ntc_pack4_desc, PACK, {})
    assert ws(l, p, P, None, P) == 0 and ws(l, None, P, None, P) == 0
    big = made(ntc.ntc_linear_desc, LINEAR, dict(num_rows=4000, num_x_rows=500))
    need = ws(big, p, P, P, P)
    assert need >= 4 * 32 * 128 * 2  # the weights in 16 bits, rows of whole lines
    assert f(big, p, P, P, P, P, P, P, None, P, P, need - 1, None) == BAD and "workspace" in ntc.ntc_last_error()
    assert f(big, p, P, P, P, P, P, P, None, P, None, need, None) == BAD
    assert f(big, p, P, P, P, P, P, P, None, P, P + 8, need, None) == BAD
    for over in (dict(in_dim=99), dict(out_dim=31), dict(type=1), dict(num_experts=3)):
        assert f(l, made(ntc.ntc_pack4_desc, PACK, over), P, P, P, P, P, P, None, P, None, 0, None) == BAD
        assert "not the layer's" in ntc.ntc_last_error()
    for bad in range(4):  # x, packed, scales, y
        a = [P] * 4
        a[bad] = None
        assert f(l, p, a[0], P, P, a[1], a[2], P, None, a[3], None, 0, None) == BAD
    assert f(l, p, P + 1, P, P, P, P, P, None, P, None, 0, None) == BAD
    assert f(l, p, P, P, P, P, P + 1, P, None, P, None, 0, None) == BAD
    assert f(l, p, P, P, P, P, P, P + 2, None, P, None, 0, None) == BAD
    assert f(l, p, P, P, None, P, P, P, None, P, None, 0, None) == BAD and "offsets" in ntc.ntc_last_error()
    assert f(l, p, P, None, P, P, P, P, None, P, None, 0, None) == BAD  # num_x_rows
    assert f(made(ntc.ntc_linear_desc, LINEAR, dict(activation=7)), p, P, P, P, P, P, P, None, P, None, 0, None) == BAD
    none = made(ntc.ntc_linear_desc, LINEAR, dict(num_rows=0, num_x_rows=0))
    assert f(none, p, None, None, P, None, None, None, None, None, None, 0, None) == OK


def test_optimizer_arguments():
    from paper_2608_27888_gb300.optim import AdamW
    with pytest.raises(ValueError, match="bits"):
        AdamW([], bits=16)
