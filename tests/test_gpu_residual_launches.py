"""Norms of more rows than one launch holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    return lib


def test_narrow_rows(g):
    """Rows of one number: the norm is its sign to 2^-11 (eps against squares of 1 and more), the 8-bit rows are the sign times 448."""
    rows = (1 << 29) + 37
    x = torch.randint(-9, 10, (rows,), device=DEV, dtype=torch.int8).to(torch.bfloat16)
    h, y = torch.full_like(x, 7.5), torch.full_like(x, 7.5)
    g.grp_rmsnorm(rows, 1, x, 1, g.DTYPE_BF16, x, 1, None, 1e-6, h, 1, y, 1, g.DTYPE_BF16)
    assert bool((h == 2 * x).all()) and bool((y == x.sign()).all())
    del h, y
    q, scale = torch.full((rows,), 3.0, device=DEV).to(torch.float8_e4m3fn), torch.full((rows + 1,), -7.0, device=DEV)
    g.grp_quantize_rows(rows, 1, x, 1, g.DTYPE_BF16, q, 1, scale)
    assert float(scale[rows]) == -7.0
    for at in range(0, rows, 1 << 27):               # (in parts: a float for every element is 2 GB)
        part = x[at:at + (1 << 27)].float()
        assert torch.equal(q[at:at + (1 << 27)].float(), part.sign() * 448)
        assert torch.equal(scale[:rows][at:at + (1 << 27)], (part.abs().double() / 448).float().clamp_min(2.0 ** -126))


def test_wide_rows(g):
    """35 GB of rows that a workgroup each takes."""
    rows, width = (1 << 24) + 3, 1032
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of device memory are needed")
    size = (torch.arange(rows, device=DEV) % 251 + 1).to(torch.bfloat16)
    x = torch.ones(rows, width, device=DEV, dtype=torch.bfloat16)
    x[:, 1::2] = -1
    x *= size[:, None]
    q, scale = torch.empty(rows, width, device=DEV, dtype=torch.float8_e4m3fn), torch.empty(rows, device=DEV)
    q.view(torch.uint8).fill_(0)
    g.grp_quantize_rows(rows, width, x, width, g.DTYPE_BF16, q, width, scale)
    assert torch.equal(scale, (size.double() / 448).float())
    bits = q.view(torch.int16)                       # two columns: 448 is 0x7E, -448 0xFE
    assert bool((bits == torch.tensor(0xFE7E - 0x10000, device=DEV, dtype=torch.int16)).all())
    del x, q, bits
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,n,k,act", [(2, 134_300_000, 8, "ACT_NONE"), (66, 67_200_001, 9, "ACT_RELU")])
def test_layers_of_many_columns(g, rows, n, k, act):
    """More columns than the kernel for few rows, or the one that keeps W in LDS, has workgroups for: tiles.  Whole numbers, so that every sum is exact."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of device memory are needed")
    r = torch.Generator(device=DEV)
    r.manual_seed(3)
    a = torch.randint(-4, 5, (rows, k), generator=r, device=DEV).to(torch.bfloat16)
    w = torch.randint(-4, 5, (k, n), generator=r, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    c = torch.full((rows, n), 0.5, device=DEV, dtype=torch.bfloat16)
    need = g.grp_linear_workspace_bytes(g.LINEAR_FORWARD, rows, n, k, g.DTYPE_BF16)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    g.grp_linear(rows, n, k, a, k, w, n, g.DTYPE_BF16, None, None, None, getattr(g, act), None, 0, c, n, g.DTYPE_BF16, None, 0, ws)
    for at in range(0, n, 1 << 25):
        want = a.float() @ w[:, at:at + (1 << 25)].float()
        want = want.relu() if act == "ACT_RELU" else want
        assert torch.equal(c[:, at:at + (1 << 25)].float(), want)          # at most 144: bf16 holds it
    del a, w, c, ws, want
    torch.cuda.empty_cache()
