"""The operators of residual blocks run together: a head of residual blocks against fp64 autograd, its training and its 8-bit serving."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    return lib


def reference(blocks, x, act):
    """The same blocks in fp64 on the weights as rounded to bf16."""
    leaves = []
    h = x.double().requires_grad_()
    leaves.append(h)
    for p, w1, w2 in zip(blocks.params, blocks.w1, blocks.w2):
        ws = [t.double().detach().requires_grad_() for t in (p[0], w1, p[2], w2, p[4])]
        leaves += ws
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + blocks.eps) * ws[0]
        h = h + act(y @ ws[1] + ws[2]) @ ws[3] + ws[4]
    return h, leaves


@pytest.mark.parametrize("rows,dim,hidden,depth", [(1, 64, 128, 1), (300, 96, 200, 3), (5000, 256, 256, 2), (77, 33, 65, 2)])
def test_blocks_against_autograd(g, rows, dim, hidden, depth):
    """Every kept tensor is rounded to bf16 (2^-9 rms 2^-9.2 of its values): some four roundings a block and pass add up, as independent ones, to less than
    2^-7 sqrt(depth) of a result's norm."""
    b = g.ResidualBlocks(dim, hidden, depth, rows, seed=3)
    r = torch.Generator(device=DEV)
    r.manual_seed(7)
    x, dout = (torch.randn(rows, dim, generator=r, device=DEV).to(torch.bfloat16) for _ in range(2))
    out = b.forward(x).clone()
    want, leaves = reference(b, x, torch.nn.functional.gelu)
    tol = 2.0 ** -7 * depth ** 0.5
    assert float((out.double() - want.detach()).norm()) <= tol * float(want.detach().norm())
    dx = b.backward(dout).clone()
    want.backward(dout.double())
    assert float((dx.double() - leaves[0].grad).norm()) <= tol * float(leaves[0].grad.norm())
    for i in range(depth):
        for got, leaf in zip(b.grads[i], leaves[1 + 5 * i:6 + 5 * i]):
            assert float((got.double() - leaf.grad).norm()) <= 2 * tol * float(leaf.grad.norm())


def test_blocks_learn(g):
    """A step lowers the loss it was made for, the gradient is clipped, and 30 of them fit a random target."""
    rows, dim = 512, 64
    b = g.ResidualBlocks(dim, 256, 2, rows, seed=1)
    r = torch.Generator(device=DEV)
    r.manual_seed(2)
    x, target = (torch.randn(rows, dim, generator=r, device=DEV).to(torch.bfloat16) for _ in range(2))
    opt = g.optimizer_desc(g.OPT_ADAM, lr=0.003)
    losses = []
    for _ in range(30):
        diff = b.forward(x).float() - target.float()
        losses.append(float(diff.square().mean()))
        b.backward((2 * diff / diff.numel()).to(torch.bfloat16))
        norm = float(b.step(opt, 0.05))
        assert abs(float(b.grad.double().norm()) - min(norm, 0.05)) <= 1e-5 * norm
    assert losses[-1] < 0.5 * losses[0]
    assert all(q < p * 1.05 for p, q in zip(losses, losses[1:]))


@pytest.mark.parametrize("rows", [1, 37, 1000])
def test_blocks_serve_in_eight_bits(g, rows):
    """Two 8-bit operands a product (2^-4 at most, rms 2^-5.8 each) against the bf16 pass: the part that the blocks add is off by less than 2^-4 of its norm."""
    b = g.ResidualBlocks(128, 512, 2, rows, act=g.ACT_SILU, seed=5)
    r = torch.Generator(device=DEV)
    r.manual_seed(4)
    x = torch.randn(rows, 128, generator=r, device=DEV).to(torch.bfloat16)
    full, served = b.forward(x).float(), b.serve(x).float()
    added = (full - x.float()).norm()
    assert float((served - full).norm()) <= 2.0 ** -4 * float(added) + 2.0 ** -8 * float(full.norm())
    assert torch.equal(b.serve(x), b.serve(x))


def test_blocks_refuse(g):
    b = g.ResidualBlocks(32, 64, 1, 10)
    for bad in (torch.zeros(11, 32, device=DEV, dtype=torch.bfloat16), torch.zeros(4, 31, device=DEV, dtype=torch.bfloat16), torch.zeros(4, 32, device=DEV),
                torch.zeros(4, 64, device=DEV, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            b.forward(bad)
    with pytest.raises(ValueError):
        g.ResidualBlocks(0, 64, 1, 10)
