"""What the operators' tests share: types, and error bounds that follow from
the arithmetic (fp32 with 24-bit significands, one rounding to the output)."""
import torch

FLOATS = [torch.float32, torch.float16, torch.bfloat16]
U32 = 2.0 ** -24  # half a unit in the last place of fp32, relative
# half a unit in the last place, relative, and half the smallest subnormal
_UNIT = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}


def rounding(ref, dtype):
    """How far one rounding of ref to dtype may be off."""
    rel, least = _UNIT[dtype]
    return ref.abs() * rel + least


def assert_within(got, ref, bound):
    """|got - ref| <= bound, element by element; ref and bound in 64 bits.  What is
    past got's type's largest number by half a unit rounds to infinity."""
    most = torch.finfo(got.dtype).max if got.dtype in _UNIT else float("inf")
    over = most * (1 + _UNIT[got.dtype][0] / 2) if got.dtype in _UNIT else most
    got, ref, bound = got.double().cpu(), ref.cpu(), bound.cpu()
    assert got.shape == ref.shape
    off = (got - ref).abs()
    infinite = got.isinf() & (got.sign() == ref.sign()) & (ref.abs() + bound >= over)
    bad = ~((off <= bound) | infinite)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} off, the worst by "
                           f"{float((off - bound)[bad].max()) if bad.any() else 0:.3g}")


def gen(seed):
    return torch.Generator().manual_seed(seed)
