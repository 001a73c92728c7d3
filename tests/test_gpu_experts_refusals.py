"""What the torch functions of the routed experts refuse: tensors of another shape, type, layout or device."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


H, I = torch.float16, torch.int32


@pytest.mark.parametrize("call,word", [
    (lambda n: n.route(z(4), 1), "two dimensions"),
    (lambda n: n.route(z(4, 8, dtype=torch.float64), 1), "float32, float16 or bfloat16"),
    (lambda n: n.route(z(8, 4).t(), 1), "last dimension"),
    (lambda n: n.route(z(1, 8).expand(4, 8), 1), "overlapping"),
    (lambda n: n.route(z(4, 8), -1), "out of range"),
    (lambda n: n.route(z(4, 8), 2, bias=z(7)), "shape"),
    (lambda n: n.route(z(4, 8), 2, bias=z(8, dtype=H)), "must be Float"),
    (lambda n: n.route(z(4, 8), 2, bias=z(16)[::2]), "contiguous"),
    (lambda n: n.route(z(4, 8), 2, bias=torch.zeros(8)), "on cuda"),
    (lambda n: n.route_backward(z(4, 8), z(4, 2), z(4, 2)), "must be Int"),
    (lambda n: n.route_backward(z(4, 8), z(4, 2, dtype=I), z(4, 3)), "shape"),
    (lambda n: n.expert_order(z(4, 2, dtype=I), 0), "num_experts"),
    (lambda n: n.expert_order(z(4, 2, dtype=I), 1025), "num_experts"),
    (lambda n: n.expert_order(z(4, 2), 4), "must be Int"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(8, dtype=H)), "two or three"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 8)), "w must be Half"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 9, dtype=H)), "shape"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(8, 3, dtype=H).t()), "last dimension"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 8, dtype=H), z(4)), "shape"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(2, 3, 8, dtype=H), offsets=z(2, dtype=I)), "shape"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 8, dtype=H), rows=z(4, 1, dtype=I)), "one dimension"),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 8, dtype=H), residual=z(3, 3, dtype=H)), "shape"),
    (lambda n: n.linear_backward(z(5, 3, dtype=H), z(4, 8, dtype=H), z(3, 8, dtype=H), activation="gelu"), "needs z"),
    (lambda n: n.linear_backward(z(4, 4, dtype=H), z(4, 8, dtype=H), z(3, 8, dtype=H)), "shape"),
    (lambda n: n.combine(z(4, 8), z(2, 2)), "must be Int"),
    (lambda n: n.combine(z(4, 8), z(2, 2, dtype=I), z(2, 3)), "shape"),
    (lambda n: n.combine(z(4, 8), z(2, 2, dtype=I), residual=z(2, 9)), "shape"),
    (lambda n: n.combine_backward(z(3, 8), z(4, 8), z(2, 2, dtype=I)), "shape")])
def test_wrong_tensors(ntc, call, word):
    with pytest.raises(ValueError, match=word):
        call(ntc)


@pytest.mark.parametrize("call,word,status", [
    (lambda n: n.route(z(4, 8), 9), "top_k", 1), (lambda n: n.route(z(4, 8), 0), "top_k", 1),
    (lambda n: n.route(z(4, 8), 2, groups=3), "num_groups", 1),
    (lambda n: n.route(z(4, 8), 2, scale=float("nan")), "scale", 1),
    (lambda n: n.linear(z(4, 8), z(3, 8)), "fp16 or bf16", 2),
    (lambda n: n.linear(z(4, 8, dtype=H), z(2, 3, 8, dtype=H)), "offsets", 1),
    (lambda n: n.linear(z(4, 8, dtype=H), z(3, 8, dtype=H), leaky_slope=float("inf")), "leaky_slope", 1)])
def test_what_the_library_refuses(ntc, call, word, status):
    with pytest.raises(ntc.NtcError, match=word) as e:
        call(ntc)
    assert e.value.status == status
