"""Products in 8-bit floating point at the ends of their sizes, on the GPU: sums of small whole
numbers, which single precision holds exactly, whatever the form adds first."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.fixture(scope="module")
def qlm():
    from paper_2407_00047_amd import qlm
    return qlm


def signs(torch, rows, blocks, seed):
    """-1, 0 or 1 for each row and block of inputs."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-1, 2, (rows, blocks), generator=gen, device="cuda", dtype=torch.int8)


def codes(torch, x):
    """The bytes of -1, 0 and 1 in e4m3."""
    return torch.where(x == 0, 0, torch.where(x > 0, 0x38, 0xb8)).to(torch.uint8)


@pytest.mark.parametrize("rows,outs", [(256, 256), (300, 64), (70, 400)])
@pytest.mark.parametrize("ins", [(1 << 23) + 1, 1 << 24])
def test_the_longest_inputs(torch, qlm, rows, outs, ins):
    """Every input of a block has its row's sign: a block's sum is 128 times the product of two signs
    (less in a last block that is not whole), and all of them together at most 2^24."""
    blocks = -(-ins // 128)
    x, w = signs(torch, rows, blocks, 1), signs(torch, outs, blocks, 2)
    tiles = -(-rows // 16)
    full = torch.zeros((16 * tiles, blocks), dtype=torch.uint8, device="cuda")
    full[:rows] = codes(torch, x)
    full = full.view(tiles, 16, blocks).transpose(1, 2)[:, :, None, :, None]
    full = full.expand(tiles, blocks, 8, 16, 16).contiguous()
    last = torch.arange(128, device="cuda").view(8, 1, 16) < ins - 128 * (blocks - 1)
    full[:, -1] *= last.to(torch.uint8)
    coded = qlm.F8Rows(full.view(torch.float8_e4m3fn),
                       torch.ones((blocks, 16 * tiles), device="cuda"), rows, ins)
    wide = codes(torch, w).repeat_interleave(128, 1)[:, :ins].contiguous()
    weight = qlm.f8_pack(wide.view(torch.float8_e4m3fn),
                         torch.ones((-(-outs // 128), blocks), device="cuda"))
    del wide
    got = qlm.f8_matmul(coded, weight, dtype=torch.float32)
    size = torch.full((blocks,), 128.0, dtype=torch.float64, device="cuda")
    size[-1] = ins - 128 * (blocks - 1)
    want = (x.double() * size) @ w.double().t().contiguous()
    assert torch.equal(got.double(), want), int((got.double() != want).sum())


def test_many_outputs(torch, qlm):
    """More than 2^34 outputs of few inputs each: the whole numbers up to 100 that they are, in
    bfloat16 too."""
    rows, outs, ins = 131077, 131073, 100
    x, w = signs(torch, rows, ins, 3), signs(torch, outs, ins, 4)
    coded = qlm.f8_rows(x.bfloat16())
    weight = qlm.f8_pack(codes(torch, w).view(torch.float8_e4m3fn),
                         torch.ones((-(-outs // 128), 1), device="cuda"))
    got = qlm.f8_matmul(coded, weight)
    other = w.float().t().contiguous()
    for at in range(0, rows, 8192):
        part = got[at:at + 8192]
        assert torch.equal(part, (x[at:at + 8192].float() @ other).bfloat16()), at
