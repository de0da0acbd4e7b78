"""Activation checkpoints in 8 bits against their definition, which is in fp32 arithmetic: codes and scales are equal, not close."""
import pytest
import torch

from test_gpu_layer import wcc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

SHAPES = [(1,), (5,), (1, 1), (3, 127), (3, 128), (3, 129), (7, 257), (2, 3, 5, 16), (9, 64), (5, 70), (33, 320), (1000, 1), (17, 8192), (4, 1000), (301, 96),
          (4096, 256), (3, 100003), (50000, 3), (777, 31), (5, 7), (100, 17), (64, 33)]
DTYPES = [torch.float32, torch.bfloat16]


def _definition(x):
    """Codes as fp64 numbers and scales, block by block; fl() is the rounding to fp32."""
    v = x.double().reshape(-1, x.shape[-1])
    codes, scales = torch.zeros_like(v), []
    for b in range(0, v.shape[1], 128):
        part = v[:, b:b + 128]
        top = part.abs().amax(1, keepdim=True)
        bad = ~torch.isfinite(part).all(1, keepdim=True)
        some = (top >= 2.0 ** -100) & ~bad
        full = torch.full_like(top, 127)
        safe = torch.where(some, top, full)
        code = torch.round((part * (full / safe).float().double()).float().double())
        codes[:, b:b + 128] = torch.where(some, code, torch.zeros_like(code))
        scales.append(torch.where(bad, torch.full_like(top, float("nan")), torch.where(some, (safe / full).float().double(), torch.zeros_like(top)))[:, 0])
    return codes.reshape(x.shape), torch.stack(scales, 1).float()


def _same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


def _check(wcc, x):      # noqa: F811
    ck = wcc.checkpoint(x)
    codes, scales = _definition(x)
    assert ck.codes.dtype == torch.int8 and torch.equal(ck.codes.double(), codes)
    assert _same(ck.scales, scales)
    L = x.shape[-1]
    wide = scales.repeat_interleave(128, 1)[:, :L].reshape(x.shape)
    want = (codes.float() * wide).to(x.dtype)
    assert _same(ck.restore(), want)
    return ck


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_definition(wcc, shape, dtype):      # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn(shape, device="cuda", generator=g) * torch.exp2(4 * torch.randn(shape[:-1] + (1,), device="cuda", generator=g))).to(dtype)
    ck = _check(wcc, x)
    # what it stands for is within half a step of 127 to the largest magnitude
    err = (ck.restore().double() - x.double()).abs().reshape(-1, shape[-1])
    step = ck.scales.double().repeat_interleave(128, 1)[:, :shape[-1]]
    assert (err <= step * (0.5 + 2.0 ** -15) + (2.0 ** -8 * 128 * step if dtype == torch.bfloat16 else 0)).all()
    assert wcc.last_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_ends_and_zeros(wcc, dtype):      # noqa: F811
    x = torch.zeros((8, 300), device="cuda")
    x[0, :128] = torch.arange(128, device="cuda") / 2                  # halves of the step: ties go to even
    x[1] = -x[0]
    x[2, 130] = 2.0 ** -101                                             # too small to keep
    x[3, 5], x[3, 6] = 2.0 ** -100, -2.0 ** -101
    x[4, 299], x[4, 0] = 3e38, 1e30
    x[5, :] = 7.0
    x[6, 128:256] = torch.linspace(-1, 1, 128, device="cuda")
    _check(wcc, x.to(dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [300, 256, 33])
def test_what_is_not_finite_takes_its_block(wcc, dtype, L):      # noqa: F811
    x = torch.ones((6, L), device="cuda", dtype=dtype)
    x[0, 0], x[1, L - 1], x[2, L // 2], x[3, 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    x[3, 2] = float("inf")
    back = _check(wcc, x).restore()
    assert torch.isnan(back[0, :min(128, L)]).all() and torch.isnan(back[1, (L - 1) // 128 * 128:]).all()
    assert (back[4:] == 1).all()


def test_other_type_out_given_room_and_stream(wcc):      # noqa: F811
    x = torch.randn((37, 200), device="cuda")
    ck = wcc.checkpoint(x)
    room = wcc.Checkpoint.like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert wcc.checkpoint(x, into=room) is room
        out = torch.full_like(x, 9)
        assert room.restore(out=out) is out
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(room.codes, ck.codes) and torch.equal(room.scales, ck.scales) and torch.equal(out, ck.restore())
    half = wcc.Checkpoint(ck.codes, ck.scales, torch.bfloat16)
    assert torch.equal(half.restore(), ck.restore().bfloat16())


def test_captured_and_replayed(wcc):      # noqa: F811
    x = torch.randn((70, 333), device="cuda")
    ck, out = wcc.Checkpoint.like(x), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wcc.checkpoint(x, into=ck).restore(out=out)
    for seed in range(3):
        x.copy_(torch.randn((70, 333), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        assert torch.equal(out, wcc.checkpoint(x).restore())


def test_neighbours_stay(wcc):      # noqa: F811
    """Codes, scales and output end where they should."""
    x = torch.randn((5, 77), device="cuda")
    codes = torch.full((5 * 77 + 64,), 55, dtype=torch.int8, device="cuda")
    scales = torch.full((5 + 8,), 55.0, device="cuda")
    ck = wcc.checkpoint(x, into=wcc.Checkpoint(codes[:5 * 77].view(5, 77), scales[:5].view(5, 1), torch.float32))
    out = torch.full((5 * 77 + 16,), 55.0, device="cuda")
    ck.restore(out=out[:5 * 77].view(5, 77))
    assert (codes[5 * 77:] == 55).all() and (scales[5:] == 55).all() and (out[5 * 77:] == 55).all()


def test_refusals(wcc):      # noqa: F811
    x = torch.randn((6, 40), device="cuda")
    ck = wcc.Checkpoint.like(x)
    bad = [lambda: wcc.checkpoint(x.t()), lambda: wcc.checkpoint(x[:, ::2]), lambda: wcc.checkpoint(x[:0]), lambda: wcc.checkpoint(x[:3], into=ck),
           lambda: wcc.checkpoint(x.bfloat16(), into=ck), lambda: ck.restore(out=x.bfloat16()), lambda: ck.restore(out=x[:5]),
           lambda: wcc.Checkpoint(ck.codes, ck.scales[:5], x.dtype), lambda: wcc.Checkpoint(ck.codes.float(), ck.scales, x.dtype)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: wcc.checkpoint(x.double()), lambda: wcc.Checkpoint(ck.codes, ck.scales, torch.float16)):
        with pytest.raises(TypeError):
            call()
    y = torch.zeros((6 * 40 + 1,), device="cuda")[1:].view(6, 40)       # 4 bytes off
    with pytest.raises(wcc.WccError) as e:
        wcc.checkpoint(y)
    assert e.value.code == 6


def test_beyond_32_bits(wcc):      # noqa: F811
    rows, L = (1 << 31) // 96 + 7, 96                                    # 2^31 and more values
    x = torch.zeros((rows, L), device="cuda", dtype=torch.bfloat16)
    x[-3:] = torch.randn((3, L), device="cuda").bfloat16()
    ck = wcc.checkpoint(x)
    want = wcc.checkpoint(x[-3:].clone())
    assert torch.equal(ck.codes[-3:], want.codes) and torch.equal(ck.scales[-3:], want.scales)
    assert not ck.scales[:-3].any()
    del x
    assert torch.equal(ck.restore()[-3:], want.restore())
