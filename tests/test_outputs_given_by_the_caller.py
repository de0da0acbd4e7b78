"""Maps that a caller hands to a layer, a chain or a block: too small, of another type, strided or elsewhere, they are refused before anything is
launched (the kernels go by the sizes of the call, so a small one would be written behind its end)."""
import pytest
import torch

from paper_2205_12268_b200 import wcc as binding


class Fake:
    """What the check looks at, without a GPU."""

    def __init__(self, n, dtype=torch.float32, device="cuda:0", contiguous=True):
        self.n, self.dtype, self.device, self.contiguous = n, dtype, torch.device(device), contiguous
        self.is_cuda = self.device.type == "cuda"

    def numel(self):
        return self.n

    def is_contiguous(self):
        return self.contiguous


@pytest.mark.parametrize("bad", [Fake(99), Fake(0), Fake(100, torch.bfloat16), Fake(100, device="cuda:1"), Fake(100, device="cpu"), Fake(100, contiguous=False)])
def test_refused(bad):
    with pytest.raises(ValueError):
        binding._room(bad, 100, Fake(100), "y")


def test_taken():
    binding._room(Fake(100), 100, Fake(7), "y")
    binding._room(Fake(101), 100, Fake(7), "y")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_through_the_entry_points(dtype):
    from paper_2205_12268_b200 import build
    from paper_2205_12268_b200 import wcc
    build.build()
    N, C, E, H, W, k = 2, 16, 40, 16, 32, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)      # noqa: E731
    x, up, down, dw = rnd(N, C, H, W).to(dtype), rnd(E, C), rnd(C, E), rnd(E, 3, 3)
    other = torch.bfloat16 if dtype == torch.float32 else torch.float32
    ad = wcc.Adapters((rnd(2, 4, E) / 6).to(dtype), rnd(2, C, 4).to(dtype))
    ids = torch.zeros((N,), dtype=torch.int32, device="cuda")
    calls = [(lambda x, y: wcc.forward(x, up, 2, k, y=y), E), (lambda x, y: wcc.Chain(x0, [up, down], 2, k)(x, y), C),
             (lambda x, y: wcc.Chain(x0, [up, down], 2, k, norms=[(None, None, 1e-5), None])(x, y), C),
             (lambda x, y: wcc.Chain(x0, [up, down], 2, k, adapters=[None, ad])(x, y, ids=ids), C), (lambda x, y: wcc.Block(x0, up, dw, down, 2, k)(x, y), C)]
    x0 = x
    for call, Cout in calls:
        want = call(x, None)
        good = torch.empty((N, Cout, H, W), device="cuda", dtype=dtype)
        assert torch.equal(call(x, good), want)
        launches = wcc.kernel_launches()
        for bad in (good[:1].clone(), good.to(other), good.cpu(), good.transpose(2, 3), torch.empty((0,), device="cuda", dtype=dtype)):
            with pytest.raises(ValueError):
                call(x, bad)
        assert wcc.kernel_launches() == launches
    for call, _ in calls[1:]:
        launches = wcc.kernel_launches()
        for bad in (x[:1].clone(), x.to(other), x.transpose(2, 3)):
            with pytest.raises(ValueError):
                call(bad, None)
        assert wcc.kernel_launches() == launches
    assert wcc.last_status() == 0
