"""What the head of residual blocks keeps between its calls, on the CPU: the operators are stood in for by plain torch, called as the library is."""
import pytest
import torch

from paper_2602_01872_amd import binding
from paper_2602_01872_amd.residual import ResidualBlocks

BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


class StandIns:
    """The operators as ResidualBlocks calls them, on CPU tensors, and the workspaces they were given."""

    def __init__(self):
        self.workspaces = []

    @staticmethod
    def put(out, m, n, v):
        out.view(-1)[:m * n].view(m, n).copy_(v)

    @staticmethod
    def take(t, m, n):
        return t.reshape(-1)[:m * n].view(m, n).float()

    def rmsnorm(self, m, d, x, ldx, xt, r, ldr, w, eps, h, ldh, y, ldy, yt, scale=None, stream=None):
        v = self.take(x, m, d) + (0 if r is None else self.take(r, m, d))
        out = v * torch.rsqrt(v.square().mean(1, keepdim=True) + eps) * w
        if h is not None:
            self.put(h, m, d, v)
        if yt == binding.DTYPE_E4M3:
            s = out.abs().amax(1) / 448
            scale.copy_(s)
            out = out / s[:, None]
        self.put(y, m, d, out)

    def quantize(self, m, d, x, ldx, xt, q, ldq, scale, stream=None):
        v = self.take(x, m, d)
        scale.copy_(v.abs().amax(1) / 448)
        self.put(q, m, d, v / scale[:, None])

    def linear(self, m, n, k, a, lda, w, ldw, t, a_s, w_s, bias, act, r, ldr, c, ldc, ct, z, ldz, ws, stream=None):
        self.workspaces.append(ws)
        A = self.take(a, m, k)
        W = w.float() if t == binding.DTYPE_BF16 else (w.float() * w_s[:, None]).t()
        v = (A if a_s is None else A * a_s[:, None]) @ W + bias
        if z is not None:
            self.put(z, m, n, v)
        v = torch.relu(v) if act == binding.ACT_RELU else v
        self.put(c, m, n, v if r is None else v + self.take(r, m, n))

    def gradient(self, *args, **kw):
        self.workspaces.append(args[-1])


@pytest.fixture
def ops(monkeypatch):
    s = StandIns()
    for name, fn in [("grp_rmsnorm", s.rmsnorm), ("grp_quantize_rows", s.quantize), ("grp_linear", s.linear), ("grp_linear_dx", s.gradient),
                     ("grp_linear_dw", s.gradient), ("grp_rmsnorm_backward", s.gradient), ("grp_gradients_create", lambda grads, outs=None: None),
                     ("grp_clip_gradients", lambda *a, **k: None), ("grp_linear_workspace_bytes", lambda *a: 64), ("grp_rmsnorm_backward_workspace_bytes", lambda *a: 64)]:
        monkeypatch.setattr(binding, name, fn)

    def optimizer_step(opt, n, step, theta, grad, m, v):        # a kernel's write: torch does not see it
        theta.data.add_(0.5)

    monkeypatch.setattr(binding, "grp_optimizer_step", optimizer_step)
    return s


def make(seed=1, rows=6):
    return ResidualBlocks(16, 24, 2, rows, act=binding.ACT_RELU, seed=seed, device="cpu")


def rows_of(n, seed=5):
    return torch.randn(n, 16, generator=torch.Generator().manual_seed(seed)).to(BF16)


def results(b, x):
    return b.forward(x).clone(), b.serve(x).clone()


@pytest.mark.parametrize("write", ["theta", "slice", "params", "inference", "refresh"])
def test_loaded_parameters_are_the_ones_that_are_used(ops, write):
    a, b, x = make(1), make(2), rows_of(6)
    want = results(a, x)
    assert not torch.equal(results(b, x)[0], want[0])
    if write == "theta":
        b.theta.copy_(a.theta)
    elif write == "slice":
        half = a.theta.numel() // 2
        b.theta[:half] = a.theta[:half]
        results(b, x)
        b.theta[half:] = a.theta[half:]
    elif write == "params":
        for p, q in zip(b.params, a.params):
            for s, t in zip(p, q):
                s.copy_(t)
    elif write == "inference":
        with torch.inference_mode():
            b.theta.copy_(a.theta)
            got = results(b, x)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    else:                                    # a write that torch does not see
        b.theta.data.copy_(a.theta)
        b.refresh()
    got = results(b, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_blocks_made_in_inference_mode_take_parameters(ops):
    a, x = make(1), rows_of(6)
    want = results(a, x)
    with torch.inference_mode():
        b = make(2)
        results(b, x)
        b.theta.copy_(a.theta)
        got = results(b, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    b.theta.mul_(2)                          # and outside it
    results(b, x)


def test_parameters_are_not_replaced(ops):
    """A tensor put in a parameter's place would be multiplied and not trained."""
    b = make()
    with pytest.raises(AttributeError):
        b.theta = torch.zeros_like(b.theta)
    with pytest.raises(TypeError):
        b.params[0][1] = torch.zeros(16, 24)


def test_refresh_makes_every_copy_there_is(ops):
    """A replayed pass makes none itself."""
    a, b, x = make(1), make(2), rows_of(6)
    results(a, x), results(b, x)
    b.theta.data.copy_(a.theta)
    b.refresh()
    assert all(torch.equal(s, t) for s, t in zip(a.w1 + a.w2, b.w1 + b.w2))
    for p, q in zip(a._served, b._served):
        assert all(torch.equal(s.float(), t.float()) for u, v in zip(p, q) for s, t in zip(u, v))


def test_a_step_is_seen_by_both_passes(ops):
    b, x = make(), rows_of(6)
    before = results(b, x)
    b.step(None, 1.0)
    after = results(b, x)
    fresh = make(2)
    fresh.theta.copy_(b.theta)
    want = results(fresh, x)
    assert not torch.equal(before[0], after[0]) and not torch.equal(before[1], after[1])
    assert torch.equal(after[0], want[0]) and torch.equal(after[1], want[1])


def test_weights_are_rounded_only_when_they_changed(ops, monkeypatch):
    b, x = make(), rows_of(6)
    results(b, x)
    calls = []
    monkeypatch.setattr(binding, "grp_quantize_rows", lambda m, d, src, *a, **k: calls.append(src.dtype) or ops.quantize(m, d, src, *a, **k))
    before = [t._version for t in b.w1 + b.w2]
    results(b, x)
    assert before == [t._version for t in b.w1 + b.w2]
    assert FP32 not in calls                 # activations are rounded at every call, weights are not
    b.theta.mul_(2)
    results(b, x)
    assert calls.count(FP32) == 4
    b.theta.mul_(2)
    b.serve(x)
    results(b, x)                            # forward rounds its own copies; those in 8 bits, which serves on other streams may be reading, stay
    assert calls.count(FP32) == 8
    b.step(None, 1.0)
    results(b, x)
    assert calls.count(FP32) == 12


def test_the_weights_copies_stay_where_they_are(ops, monkeypatch):
    """A captured pass reads them at their addresses."""
    b, x = make(), rows_of(6)
    results(b, x)
    places = []
    for _ in range(2):
        seen = []
        monkeypatch.setattr(binding, "grp_linear", lambda *a, **k: seen.append(a[5].data_ptr()) or ops.linear(*a, **k))
        results(b, x)
        places.append(seen)
        b.theta.mul_(2)
    assert places[0] == places[1]


def test_no_workspace_is_kept(ops):
    """Calls that run side by side on two streams, a captured pass and a later larger one: each writes its own partial sums."""
    b = make()
    x = rows_of(6)
    b.forward(x)
    b.backward(x)
    b.serve(x[:1].contiguous())
    b.serve(x)
    own = {t.untyped_storage().data_ptr() for t in vars(b).values() if torch.is_tensor(t)}
    assert len(ops.workspaces) > 12
    for ws in ops.workspaces:
        assert ws.numel() >= 64 and ws.untyped_storage().data_ptr() not in own
    assert all(ws.untyped_storage().data_ptr() != other.untyped_storage().data_ptr() for ws in ops.workspaces[-4:] for other in ops.workspaces[:-8])


def test_backward_takes_the_rows_of_the_last_forward(ops):
    b = make(rows=10)
    with pytest.raises(ValueError):          # nothing is kept yet
        b.backward(rows_of(4))
    b.forward(rows_of(10))
    b.forward(rows_of(4))
    for n in (10, 5, 3, 0):
        with pytest.raises(ValueError):
            b.backward(rows_of(n))
    b.serve(rows_of(10))                     # keeps nothing
    b.backward(rows_of(4))
    b.backward(rows_of(4))                   # the kept rows are still there
    with pytest.raises(ValueError):          # a refused call leaves them
        b.forward(rows_of(11))
    b.backward(rows_of(4))
    b.forward(rows_of(0))
    b.backward(rows_of(0))


def test_tensors_of_another_device_are_refused(ops):
    """A kernel that is handed host memory faults."""
    b = make()
    elsewhere = torch.empty(4, 16, dtype=BF16, device="meta")
    for call in (b.forward, b.backward, b.serve):
        with pytest.raises(ValueError):
            call(elsewhere)


def test_gradients_on_the_host_are_refused():
    host = torch.zeros(8)
    with pytest.raises(ValueError):
        binding.grp_gradients_create([host])
    with pytest.raises(ValueError):
        binding.grp_gradients_create([torch.empty(8, device="meta")], [host])
    with pytest.raises(ValueError):          # an output for every tensor
        binding.grp_gradients_create([torch.empty(8, device="meta")], [])
