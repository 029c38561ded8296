"""Shared by the tests of include/xnor_lowbit.h: element types with their unit roundoff, seeded tensors, row views."""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # unit roundoff: significands of 24, 8 and 11 bits
SMALLEST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}   # subnormals round to multiples of these
EPS32 = 2.0 ** -24


def generator(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def normal(gen, *shape, scale=1.0):
    return scale * torch.randn(shape, generator=gen)


def apart(t, extra):
    """The same matrix on the GPU with its rows `extra` elements further apart (0: dense)."""
    if not extra:
        return t.cuda()
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t.cuda()
    return wide[:, :t.shape[1]]


def filled(shape, dtype):
    """An output no kernel would leave behind by chance."""
    if dtype.is_floating_point:
        return torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    return torch.full(shape, -77 if dtype != torch.uint8 else 201, dtype=dtype, device="cuda")


def assert_within(got, want, bound, what):
    """|got - want| <= bound element by element, in 64 bits; NaN and infinities have to be the same."""
    got, want = got.detach().double().cpu(), want.double().cpu()
    bound = torch.as_tensor(bound, dtype=torch.float64).expand_as(want)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, f"{what}: off by {float((got - want).abs()[fine].max()):.3g}, {int((over > 0).sum())} values"
