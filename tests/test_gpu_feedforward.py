"""The adapted feed-forward half, and the adapter with 8-bit activations, against float64 autograd of the same network,
whose activation's slope is taken at the 8-bit rounding of the pre-activation, as the layer's is by definition (relu's
jumps: a small positive value that rounds to zero has slope zero).

Gradients are taken at values rounded to 8 bits.  A block's step is at most 1/63.5 of its largest value, which for 32
normal values is 2.1 deviations on average, so the rounding has an RMS of at most 0.033 / sqrt(12) = 1 % of a value's;
the slopes are of order one, three such roundings (pre-activation, h, the norm's input) and the 16-bit ones of the
operands (at most 0.2 % each) add up to less than 2.5 %.  Bounds on rel-L2: 3e-2, and 1e-2 for y, which sees no 8 bits.
"""

import pytest
import torch

from paper_2511_01385_amd import api
from paper_2511_01385_amd.feedforward import AdaptedFeedForward
from paper_2511_01385_amd.layer import BlockCirculantLinear
from tests.test_gpu_act8 import reference

pytestmark = pytest.mark.gpu

class AtCheckpoint(torch.autograd.Function):
    """act(z) whose gradient is taken at z's 8-bit rounding."""

    @staticmethod
    def forward(ctx, z, act):
        rounded = reference(z.detach().reshape(-1, z.shape[-1]).cpu().numpy())[2]
        ctx.save_for_backward(torch.from_numpy(rounded).to(z.device).reshape(z.shape))
        ctx.act = act
        return act(z)

    @staticmethod
    def backward(ctx, g):
        with torch.enable_grad():
            z = ctx.saved_tensors[0].requires_grad_(True)
            return torch.autograd.grad(ctx.act(z), z, g)[0], None


ACTS = {"gelu": torch.nn.functional.gelu, "relu": torch.relu, "silu": torch.nn.functional.silu}


def circulant(c):
    """The dense matrix of first columns c (q, kb, p)."""
    q, kb, p = c.shape
    m = torch.arange(p, device=c.device)
    return c[:, :, (m[:, None] - m[None, :]) % p].permute(0, 2, 1, 3).reshape(q * p, kb * p)


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("tokens,d_model,d_ff,p,activation", [(333, 256, 1024, 64, "gelu"), (40, 768, 768, 256, "silu"),
                                                              (1000, 512, 512, 512, "none"), (129, 64, 192, 32, "relu")])
def test_against_float64_autograd(dtype, tokens, d_model, d_ff, p, activation):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    net = AdaptedFeedForward(d_model, d_ff, p, dtype=dtype, activation=activation)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    with torch.no_grad():
        net.b1.copy_(0.1 * rand(d_ff)), net.b2.copy_(0.1 * rand(d_model))
        net.c.copy_(rand(*net.c.shape) * 0.3 * d_ff**-0.5)
        net.weight.copy_(1 + 0.1 * rand(d_model)), net.bias.copy_(0.1 * rand(d_model))
    x = rand(2, tokens, d_model).to(dtype).requires_grad_(True)
    dy = rand(2, tokens, d_model).to(dtype)
    y = net(x)
    dx, dc, dw, db = torch.autograd.grad(y, (x, net.c, net.weight, net.bias), dy)

    d = lambda t: t.detach().double()  # noqa: E731
    x64 = d(x).requires_grad_(True)
    c64, w64, b64 = (d(t).requires_grad_(True) for t in (net.c.to(dtype), net.weight, net.bias))
    z = x64 @ d(net.w1).t() + d(net.b1)
    h = z if activation == "none" else AtCheckpoint.apply(z, ACTS[activation])
    o = h @ d(net.w2).t() + d(net.b2) + h @ circulant(c64).t() + x64
    want = torch.nn.functional.layer_norm(o, (d_model,), w64, b64, net.eps)
    grads = torch.autograd.grad(want, (x64, c64, w64, b64), d(dy))
    assert rel(y, want) < 1e-2
    for name, got, ref in zip(("dx", "dc", "dweight", "dbias"), (dx, dc, dw, db), grads):
        assert rel(got, ref) < 3e-2, (name, rel(got, ref))


def test_a_step_of_training_lowers_the_loss():
    torch.manual_seed(3)
    net = AdaptedFeedForward(256, 512, 64)
    x = torch.randn(512, 256, device="cuda").bfloat16()
    target = torch.randn(512, 256, device="cuda")
    opt = torch.optim.SGD(net.parameters(), lr=1.0)
    losses = []
    for _ in range(5):
        loss = (net(x).float() - target).square().mean()
        losses.append(float(loss))
        opt.zero_grad()
        loss.backward()
        opt.step()
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_what_is_kept_for_the_backward():
    tokens, d_model, d_ff = 4096, 1024, 4096
    net = AdaptedFeedForward(d_model, d_ff, 256)
    x = torch.randn(tokens, d_model, device="cuda").bfloat16().requires_grad_(True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = net(x)
    kept = torch.cuda.memory_allocated() - before - y.numel() * 2
    # the 8-bit checkpoints, the spectra, mean and rstd, and no activation in the storage type (a few blocks' rounding)
    held = tokens * (2 * d_ff + d_model) * 33 // 32
    spectra = net.c.numel() * 2
    assert kept <= held + spectra + 8 * tokens + 64 * 1024
    y.sum().backward()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d_in,d_out,p", [(256, 256, 64), (768, 768, 256), (512, 1024, 128), (16384, 16384, 16384)])
def test_adapter_with_8_bit_activations(dtype, d_in, d_out, p):
    torch.manual_seed(5)
    layer = BlockCirculantLinear(d_in, d_out, p, dtype=dtype, checkpoint8=True)
    plain = BlockCirculantLinear(d_in, d_out, p, dtype=dtype)
    with torch.no_grad():
        plain.c.copy_(layer.c)
    x = torch.randn(70, d_in, device="cuda").to(dtype)
    g = torch.randn(70, d_out, device="cuda").to(dtype)
    out = []
    for net in (layer, plain):
        xi = x.clone().requires_grad_(True)
        y = net(xi)
        out.append((y, *torch.autograd.grad(y, (xi, net.c), g)))
    (y8, dx8, dc8), (y, dx, dc) = out
    assert torch.equal(y8, y)
    assert torch.equal(dx8, dx)  # (dx does not depend on x)
    assert rel(dc8, dc.double()) < 2e-2


def test_second_derivatives_are_refused():
    net = AdaptedFeedForward(256, 512, 64)
    x = torch.randn(10, 256, device="cuda").bfloat16().requires_grad_(True)
    y = net(x)
    plain = torch.autograd.grad(y.float().square().sum(), x, retain_graph=True)[0]
    dx = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)[0]
    assert torch.equal(dx, plain)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.float().sum() + dx.float().square().sum()).backward()


@pytest.mark.parametrize("how", ["no_grad", "inference_mode", "frozen"])
def test_no_checkpoints_without_a_backward(how, monkeypatch):
    net = AdaptedFeedForward(256, 512, 64)
    with torch.no_grad():
        net.c.normal_(std=0.01)
    x = torch.randn(100, 256, device="cuda").bfloat16()
    want = net(x).detach()

    def closed(*args, **kwargs):
        raise AssertionError("a checkpoint was made")

    monkeypatch.setattr(api, "checkpoint_like", closed)
    monkeypatch.setattr(api, "act8_quantize", closed)
    if how == "frozen":
        net.requires_grad_(False)
        y = net(x)
    else:
        with getattr(torch, how)():
            y = net(x)
    assert not y.requires_grad and torch.equal(y, want)
    net.requires_grad_(True)
    with pytest.raises(AssertionError, match="checkpoint"):
        net(x)


@pytest.mark.parametrize("how", ["no_grad", "inference_mode", "frozen"])
def test_no_checkpoint_of_the_adapter_without_a_backward(how, monkeypatch):
    net = BlockCirculantLinear(256, 512, 64, checkpoint8=True)
    x = torch.randn(100, 256, device="cuda").bfloat16()
    want = net(x).detach()

    def closed(*args, **kwargs):
        raise AssertionError("a checkpoint was made")

    monkeypatch.setattr(api, "checkpoint_like", closed)
    monkeypatch.setattr(api, "act8_quantize", closed)
    if how == "frozen":
        net.requires_grad_(False)
        y = net(x)
    else:
        with getattr(torch, how)():
            y = net(x)
    assert not y.requires_grad and torch.equal(y, want)
    for parameter, value in ((True, False), (False, True)):
        net.requires_grad_(parameter)
        with pytest.raises(AssertionError, match="checkpoint"):
            net(x.detach().requires_grad_(value))
