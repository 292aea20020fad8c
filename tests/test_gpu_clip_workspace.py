"""The norm over many tensors and the clipping in a caller's workspace of the size that tcr.h states: 64 KiB, or 8 bytes for each 143 tensors where that is more; of a caller's buffer half of
what follows its first 256 bytes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.set_workspace(None)
    torch.cuda.empty_cache()


def small_and_large(small, large, elements):
    """`small` tensors of one element behind each other, `large` ones of `elements` behind them, 5 small ones."""
    room = torch.randn(small + 5, device="cuda")
    more = torch.randn(large * elements, device="cuda").to(torch.bfloat16)
    return [room[i:i + 1] for i in range(small)] + [more[i * elements:(i + 1) * elements] for i in range(large)] + [room[small + i:small + i + 1] for i in range(5)]


@pytest.mark.parametrize("small,large,elements", [(0, 1, 8192 * 8192 + 1), (0, 3, 8192 * 9000), (2000, 143, 8192 * 130), (429, 1, 8192 * 20000), (0, 0, 0), (8188, 0, 0), (0, 143, 8192 * 57)], ids=str)
def test_the_stated_workspace_is_enough(tcr, small, large, elements):
    tensors = small_and_large(small, large, elements)
    want = torch.stack([t.double().square().sum() for t in tensors[small:]] + [torch.cat(tensors[:small] or [torch.zeros(1, device="cuda")]).double().square().sum()]).sum().sqrt()
    usual = tcr.gradient_norm(tensors)
    room = torch.empty(256 + 2 * (64 << 10), dtype=torch.uint8, device="cuda")
    tcr.set_workspace(room)
    try:
        got = tcr.gradient_norm(tensors)
        assert torch.equal(got, usual) and abs(float(got) - float(want)) <= 2.0 ** -23 * float(want)
        other = [torch.empty_like(t) for t in tensors]
        assert torch.equal(tcr.clip_gradients(tensors, 0.5 * float(want), out=other), got)
        factor = 0.5 * float(want) / (float(want) + 1e-6)
        # (the roundings of the factor, of the product and of the type)
        for t, o in zip(tensors[-9:], other[-9:]):
            eps = 2.0 ** -23 + (0.0 if o.dtype == torch.float32 else torch.finfo(o.dtype).eps / 2)
            assert ((o.double() - factor * t.double()).abs() <= eps * t.double().abs() + 2.0 ** -126).all()
    finally:
        tcr.set_workspace(None)


def test_many_small_tensors_beside_large_ones(tcr):
    """101 launches, of which all but one would have less than one workgroup's share of the sums; a tensor may be listed more than once where nothing is written."""
    large, small = torch.randn(8192 * 10000, device="cuda").to(torch.bfloat16), torch.randn(143, device="cuda")
    tensors = [large] * 143 + [small[i:i + 1] for i in range(143)] * 100
    want = float(143 * large.double().square().sum() + 100 * small.double().square().sum()) ** 0.5
    tcr.set_workspace(torch.empty(256 + 2 * (64 << 10), dtype=torch.uint8, device="cuda"))
    try:
        assert abs(float(tcr.gradient_norm(tensors)) - want) <= 2.0 ** -23 * want
    finally:
        tcr.set_workspace(None)


def test_with_less_nothing_is_done(tcr):
    tensors = small_and_large(0, 2, 8192 * 8192)
    before = tensors[0][:1000].clone()
    tcr.set_workspace(torch.empty(256 + (64 << 10), dtype=torch.uint8, device="cuda"))
    try:
        with pytest.raises(tcr.TcrError) as e:
            tcr.clip_gradients(tensors, 1.0)
        assert e.value.status == tcr.ERR_WORKSPACE and torch.equal(tensors[0][:1000], before)
    finally:
        tcr.set_workspace(None)
