"""The codes of the norm in 8 bits are what the header says: the binary32 quotient of the norm and its scale, rounded to nearest even.  The norm of binary32
rows is what rms_norm gives for them, bit for bit, so codes and scales have one right value each: no tolerance."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def expected(y, scales, group, kind):
    """By the CPU's division and rounding."""
    cols = y.shape[1]
    y, scales = y.cpu(), scales.cpu()
    quotient = y / scales.repeat_interleave(group or cols, 1)[:, :cols]
    return quotient.to(kind) if kind == torch.float8_e4m3fn else quotient.round().to(torch.int8)


@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("rows,cols", [(60000, 64), (8000, 512), (4000, 1024), (1000, 5120), (200, 20000)])
def test_codes_are_rounded_quotients(tcr, kind, group, rows, cols):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cols)
    # (values of few bits and a weight of one: quotients fall on the middle between two codes)
    x = torch.randn(rows, cols, generator=gen, device="cuda").bfloat16().float()
    w = torch.ones(cols, device="cuda")
    y = tcr.rms_norm(x, w)
    codes, scales = tcr.rms_norm_quantized(x, w, dtype=kind, group=group)
    parts = torch.nn.functional.pad(y, (0, -cols % (group or cols))).view(rows, -1, group or cols)
    assert torch.equal(scales.cpu(), parts.abs().amax(2).cpu() / (448.0 if kind == torch.float8_e4m3fn else 127.0))
    want = expected(y, scales, group, kind)
    assert (codes.cpu().view(torch.uint8) != want.view(torch.uint8)).sum().item() == 0


@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
def test_codes_of_extreme_scales(tcr, kind):
    # scales from the least, 2^-126, to 2^119: weights bring the norm there
    x = torch.randn(4, 256, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    for power in (-149, -140, -126, -120, -118, -60, 0, 60, 100, 124, 125):
        w = torch.full((256,), 2.0 ** power, device="cuda")
        y = tcr.rms_norm(x, w)
        codes, scales = tcr.rms_norm_quantized(x, w, dtype=kind)
        assert (scales >= 2.0 ** -126).all() and torch.isfinite(scales).all()
        assert torch.equal(codes.cpu().view(torch.uint8), expected(y, scales, 0, kind).view(torch.uint8)), power


@pytest.mark.parametrize("group", [0, 32])
def test_an_infinite_norm(tcr, group):
    # an infinity in the weight: its column has no code, the others of its group are 0 beside it
    x = torch.ones(3, 96, device="cuda")
    w = torch.ones(96, device="cuda")
    w[40] = float("inf")
    codes, scales = tcr.rms_norm_quantized(x, w, group=group)
    beside = torch.ones(96, dtype=torch.bool, device="cuda") if group == 0 else torch.arange(96, device="cuda") // group == 1
    beside[40] = False
    assert torch.isnan(codes[:, 40].float()).all() and (codes[:, beside].float() == 0).all()
    assert torch.isinf(scales).sum().item() == 3
    codes, _ = tcr.rms_norm_quantized(x, w, group=group, dtype=torch.int8)
    assert (codes[:, beside] == 0).all() and (codes[:, 40] == 0).all()
