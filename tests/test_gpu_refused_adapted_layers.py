"""A layer with adapters that is refused has launched nothing: y, which may be the caller's residual too, keeps what it held."""
import pytest
import torch

from test_gpu_adapted_layers import _made
from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(3, 24, 40, 16, 32, 2, 8), (2, 300, 400, 8, 16, 2, 12)])
def test_a_refused_layer_leaves_its_output(wcc, shape, dtype):      # noqa: F811
    N, Cin, Cout, H, W, R, r = shape
    d = _made(*shape, dtype)
    ad, ids = wcc.Adapters(d["A"], d["B"], d["scale"]), d["ids"]
    ids[0] = 1
    bad = [(dict(k=0), wcc.WccError), (dict(k=H * W + 1), wcc.WccError), (dict(bits=1), wcc.WccError), (dict(levels=4), wcc.WccError),
           (dict(ws=wcc.Workspace(1024, "cuda")), wcc.WccError), (dict(alpha=float("inf")), wcc.WccError), (dict(wbits=9), wcc.WccError),
           (dict(Wt=d["Wt"].to(torch.bfloat16)), TypeError), (dict(Wt=d["Wt"][:, :8].contiguous()), ValueError), (dict(ids=ids.long()), ValueError),
           (dict(residual=d["res"][:, :8].contiguous()), ValueError), (dict(Wt=None), (AttributeError, ValueError)),
           (dict(taps=("idx",), ws=wcc.Workspace(1024, "cuda")), wcc.WccError)]
    for kw, error in bad:
        y = d["res"].clone()
        call = dict(x=d["x"], Wt=d["Wt"], levels=2, k=128, bits=8, adapters=ad, ids=ids, residual=y, y=y)
        launches = wcc.kernel_launches()
        with pytest.raises(error):
            wcc.forward(**dict(call, **kw))
        assert wcc.kernel_launches() == launches, kw
        assert torch.equal(y, d["res"]), kw
    y = d["res"].clone()
    assert torch.equal(wcc.forward(d["x"], d["Wt"], 2, 128, adapters=ad, ids=ids, residual=y, y=y),
                       wcc.forward(d["x"], d["Wt"], 2, 128, adapters=ad, ids=ids, residual=d["res"]))
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_workspace_of_the_layer_serves_its_adapters(wcc, dtype):      # noqa: F811
    """Factors too large for shared memory are laid out in the caller's workspace where it has the room; a smaller one still serves the layer."""
    d = _made(2, 400, 300, 8, 16, 3, 40, dtype, 3)
    ad = wcc.Adapters(d["A"], d["B"], d["scale"])
    least = wcc.Workspace.for_problem(d["x"], 300, 2, 32, 8)
    need = ad.workspace(d["x"], backward=False).nbytes
    want = wcc.forward(d["x"], d["Wt"], 2, 32, residual=ad(d["x"], d["ids"]))
    for nbytes in (least.nbytes, max(need, least.nbytes), 4 * max(need, least.nbytes)):
        ws = wcc.Workspace(nbytes, "cuda")
        for _ in range(2):
            assert torch.equal(wcc.forward(d["x"], d["Wt"], 2, 32, adapters=ad, ids=d["ids"], ws=ws), want)
    assert wcc.last_status() == 0
