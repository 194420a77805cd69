"""Calls of very many clients: right up to 2^32 threads a launch, refused from there on, since the device would run what is left of their number
in 32 bits and say nothing."""
import pytest
import torch

from test_gpu_ops_linear import DEV, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(ops, n):   # noqa: F811
    """Of n clients with a value each: the outputs, and what each of them is everywhere."""
    x = torch.full((n, 1, 1), 3.0, device=DEV)
    code, scale = (torch.full((n, 1, 1), v, dtype=torch.uint8, device=DEV) for v in (5, 126))   # 3 times 2^-1
    zero, one = torch.zeros(n, 1, device=DEV), torch.ones(n, 1, device=DEV)
    maps = x[:, :, None]
    return {
        "linear": lambda: (ops.aet_linear_forward(x, x)[0], 9.0),
        "linear gradient": lambda: (*ops.aet_linear_backward(x, x, x), 9.0, 9.0, 3.0),
        "group norm": lambda: (ops.aet_group_norm_forward(maps, 1)[0], 0.0),
        "group norm gradient": lambda: (*ops.aet_group_norm_backward(maps, maps, zero[:, None], one[:, None], one, zero)[1:], 9.0, 3.0),
        "dropout": lambda: (ops.aet_dropout_forward(x, p=0.0, seed=1), 3.0),
        "layer norm": lambda: (ops.aet_layer_norm_forward(x, beta=one)[0], 1.0),
        "layer norm gradient": lambda: (*ops.aet_layer_norm_backward(x, x, zero, one, one), -27.0, 9.0, 3.0),
        "quantise": lambda: (*ops.aet_mx4_quantise(x), 7, 126),
        "dequantise": lambda: (ops.aet_mx4_dequantise(code, scale, cols=1, dtype=torch.float32), 1.5),
        "4-bit linear": lambda: (ops.aet_mx4_linear_forward(code, scale, code, scale, cols=1, dtype=torch.float32)[0], 2.25),
        "4-bit linear gradient": lambda: (*ops.aet_mx4_linear_backward(x, code, scale, code, scale, cols=1), 4.5, 4.5, 3.0),
        "sums over no rows": lambda: (*ops.aet_layer_norm_backward(x[:, :0], x[:, :0], zero[:, :0], one[:, :0], one)[1:], 0.0, 0.0),
    }


@pytest.mark.parametrize("n", [(1 << 22) - 1, (1 << 24) - 3, (1 << 24) + 8], ids=str)
def test_many_clients(ops, n):   # noqa: F811
    from paper_2112_13935_amd import AetError
    refused = []
    for name, call in calls(ops, n).items():
        try:
            out = call()
        except AetError as e:
            assert "2^32" in str(e), name
            refused.append(name)
            continue
        got, want = out[:len(out) // 2], out[len(out) // 2:]
        assert all(bool((t == v).all()) for t, v in zip(got, want)), name
    if n < 1 << 22:
        assert not refused
    if n > 1 << 24:
        assert {"quantise", "dequantise", "layer norm gradient", "4-bit linear", "4-bit linear gradient", "linear gradient"} <= set(refused)
