"""How far products with weights in 4 bits are off what 64 bits give, all elements together, for activations with and without a mean.

What the kernels may lose (variances, for codes q that are even over -7..7 and independent of x).  A rounding in 32 bits of a sum of size t adds
at most 2^-48 t^2 / 3.  In a group there are `adds` sums a product.  What is added to the codes and taken away again takes them up to lift * sum |x| and
back, each on average a third of that squared; the sum itself has a square of at most mean q^2 * sum x^2; a factor of 2 covers the two together.  Over
the width there are two roundings a group and 16 for the wavefronts, of at most the whole sum.  To that comes the result's own rounding, which is measured."""
import numpy as np
import pytest
import torch

DEV = "cuda:0"
LIFT = {torch.float32: 0, torch.bfloat16: 136, torch.float16: 72}
ADDS = {torch.float32: 3, torch.bfloat16: 2, torch.float16: 2}       # fp32: x in three parts; else the codes' products and what is taken away
Q2 = 7 * 8 / 3                                               # mean square of a code


def activations(kind, m, k, g):
    x = torch.randn(m, k, generator=g, device=g.device)
    return {"centred": x, "magnitudes": x.abs(), "behind a ReLU": x.clamp(min=0), "offset": x + 3}[kind]


KINDS = ["centred", "magnitudes", "behind a ReLU", "offset"]


def weights(n, k, group, g):
    """Even codes of -7..7 (nibbles [n][k]) and scales of 1/2 to 2."""
    q = torch.randint(-7, 8, (n, k), generator=g, device=g.device)
    s = torch.exp2(2 * torch.rand(n, -(-k // group), generator=g, device=g.device) - 1).to(torch.bfloat16)
    return q, s


def allowed(x, s, group, lift, adds):
    """The sum over all results of the variances above."""
    m, k = x.shape
    pad = torch.nn.functional.pad(x.double(), (0, s.shape[1] * group - k)).view(m, -1, group)
    ones, twos, s2 = pad.abs().sum(2), pad.square().sum(2), s.double().square().t().contiguous()
    inside = adds * group * 2 * ((lift * lift / 3 * ones.square() + Q2 * twos) @ s2)
    across = (2 * s.shape[1] + 16) * Q2 * (twos @ s2)
    return (2.0 ** -48 / 3 * (inside + across)).sum().item()


def exact(x, q, s, group):
    return x.double() @ (q.double() * s.double().repeat_interleave(group, 1)[:, :q.shape[1]]).t().contiguous()


def off(y, want, x, s, group, lift, adds):
    """The error of all results together over what it may be.  (3 %: both are taken from the same few thousand results.)"""
    rounding = (want.to(y.dtype).double() - want).square().sum().item()
    return ((y.double() - want).square().sum().item() / (rounding + allowed(x, s, group, lift, adds))) ** 0.5 / 1.03


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (3, 2000, 1000), (13, 700, 2043), (24, 333, 4000), (150, 130, 2048), (600, 2100, 520)])
@pytest.mark.parametrize("kind", KINDS)
def test_products(dtype, group, m, n, k, kind):
    from paper_2009_13003_amd import lc
    g = torch.Generator(device=DEV); g.manual_seed(m + n + k + group)
    q, s = weights(n, k, group, g)
    x = activations(kind, m, k, g).to(dtype)
    codes = torch.full((n, lc.lc_w4_row_bytes(k)), 0x88, dtype=torch.uint8, device=DEV)
    c = torch.nn.functional.pad((q + 8).to(torch.uint8), (0, k % 2), value=8)
    codes[:, :c.shape[1] // 2] = c[:, 0::2] | c[:, 1::2] << 4
    y = lc.lc_w4_matmul(x, lc.W4(codes, s, k, group))
    assert off(y, exact(x, q, s, group), x, s, group, LIFT[dtype], ADDS[dtype]) <= 1


def emulated(x, q, s, group, lift, parts):
    """A product's sums in 32 bits, one element of the width after another: what is added to the codes is taken away first; fp32 x in `parts` parts
    of a bf16's leading bits, the least first."""
    m, k = x.shape
    left, total, of = x.float().numpy(), np.zeros((m, q.shape[0]), np.float32), []
    if parts:
        for _ in range(parts):
            of.append((left.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32))
            left = left - of[-1]
    else:
        of = [left]
    q = q.numpy().astype(np.float32)
    for b in range(0, k, group):
        acc = np.zeros_like(total)
        for j in range(b, min(k, b + group)):
            if lift:
                acc = acc - (np.float32(lift) * of[0][:, j])[:, None]
        for p in reversed(of):
            for j in range(b, min(k, b + group)):
                acc = acc + p[:, j][:, None] * (q[:, j] + np.float32(lift))[None]
        total = total + acc * s.float().numpy()[:, b // group][None]
    return torch.from_numpy(total)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("kind", KINDS)
def test_the_bound_tells_them_apart(group, kind):
    """On the CPU: the arithmetic above keeps the bound, fp32 in two parts does not, nor fp16 whose codes are raised by 1032 where x has a mean."""
    m, n, k = 32, 128, 1024
    g = torch.Generator(); g.manual_seed(group)
    q, s = weights(n, k, group, g)
    x = activations(kind, m, k, g)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        t = x.to(dtype)
        want = exact(t, q, s, group)
        parts = 3 if dtype == torch.float32 else 0
        assert off(emulated(t, q, s, group, LIFT[dtype], parts).to(dtype), want, t, s, group, LIFT[dtype], ADDS[dtype]) <= 1
        if parts:
            assert off(emulated(t, q, s, group, 0, 2), want, t, s, group, 0, 3) > 1.5
        if dtype == torch.float16 and kind != "centred" and group == 128:
            assert off(emulated(t, q, s, group, 1032, 0).to(dtype), want, t, s, group, 72, 2) > 1
