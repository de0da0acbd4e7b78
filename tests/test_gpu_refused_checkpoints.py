"""A backward pass on a checkpoint that the binding refuses has launched nothing: the checkpoint is brought back only once its arguments are right."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def test_nothing_is_launched(wcc):      # noqa: F811
    x = torch.randn((2, 16, 8, 12), device="cuda")
    ck = wcc.checkpoint(x)
    _, mean, rstd = wcc.layernorm(x, stats=True)
    ad = wcc.Adapters(torch.randn((2, 4, 16), device="cuda"), torch.randn((2, 16, 4), device="cuda"))
    ids = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    rows = torch.randn((40, 16), device="cuda").bfloat16()
    kept = wcc.checkpoint(rows)
    W = torch.randn((24, 16), device="cuda").bfloat16()
    dy = torch.randn((40, 24), device="cuda").bfloat16()
    bad = [lambda: wcc.layernorm_backward(x[:1], ck, mean, rstd), lambda: wcc.layernorm_backward(x, ck, mean[:1], rstd),
           lambda: wcc.layernorm_backward(x, ck, mean, rstd, dx=x[:1]), lambda: ad.backward(x[:1], ck, ids), lambda: ad.backward(x, ck, ids[:1]),
           lambda: ad.backward(x, ck, ids, dx=x), lambda: wcc.gated_backward(dy[:39], kept, W, W), lambda: wcc.gated_backward(dy, kept, W, W[:16]),
           lambda: wcc.gated_backward(dy, kept, W, W, act="tanh"), lambda: wcc.gated_backward(dy, kept, W, W, dx=dy)]
    for i, call in enumerate(bad):
        launches = wcc.kernel_launches()
        with pytest.raises(ValueError):
            call()
        assert wcc.kernel_launches() == launches, i
    launches = wcc.kernel_launches()
    with pytest.raises(TypeError):
        wcc.gated_backward(x, ck, W, W)
    assert wcc.kernel_launches() == launches
