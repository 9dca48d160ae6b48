"""Errors of the calls on either cache name the call that was made."""
import pytest
import torch

from paper_1705_09864_amd import binding as B


def calls(bits):
    return ("kv4_write", "kv4_read", "kv4_attention") if bits == 4 else ("kv_write", "kv_read", "kv_attention")


@pytest.mark.parametrize("bits", [8, 4])
def test_not_on_the_gpu(bits):
    x, (write, _, attention) = torch.zeros((2, 3, 64)), calls(bits)
    for name, args in ((write + " k", (x, x, x, x, x, x)), (attention + " q", (x, x, x, x, x))):
        with pytest.raises(ValueError, match="^%s: tensor must live on the GPU" % name):
            getattr(B, name.split()[0])(*args)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_arguments(bits):
    write, read, attention = calls(bits)
    cache = (B.kv4_cache if bits == 4 else B.kv_cache)(3, 2, 64) + (torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.ones((1,), dtype=torch.int32, device="cuda"))
    x = torch.zeros((1, 2, 64), device="cuda")
    q = torch.zeros((1, 4, 64), device="cuda")
    for name, args, named in ((write + " k", (x.double(), x) + cache, {}), (write + " k", (x[:, :1], x) + cache, {}), (write + " v", (x, x.half()) + cache, {}),
                              (write + " v", (x, x[:, :1]) + cache, {}), (read + " dtype", cache + (64, "f16", 1), {}), (read + " dtype", cache + (64, torch.int32, 1), {}),
                              (read + " out_k", cache + (64, torch.half, 1), dict(out_k=x)), (read + " out_v", cache + (64, torch.float32, 1), dict(out_v=x[0])),
                              (read + " out_v", cache + (64, torch.float32, 1), dict(out_v=x[:, :1])), (attention + " q", (q[0],) + cache, {}),
                              (attention + " out", (q,) + cache, dict(out=q.half())), (attention + " out", (q,) + cache, dict(out=x))):
        with pytest.raises(ValueError, match="^%s: " % name):
            getattr(B, name.split()[0])(*args, **named)
    for name, args in ((read, cache + (64, torch.float32, -1)), (attention, (q[:, :3],) + cache)):
        with pytest.raises(B.BmxError, match="bmx_%s\\b" % name):
            getattr(B, name)(*args)
