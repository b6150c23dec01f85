"""Plain definitions of the microscaled 4-bit matrices, in 64 bits on the CPU."""
import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
EPS = 2.0 ** -24


def quantise(x):
    """(codes 0 to 15 of every value, scale bytes of every block) of x's rows, both
    over whole groups of 128 columns."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    v = torch.zeros(rows, groups * 128, dtype=torch.float64)
    v[:, :cols] = x.double()
    v = v.view(rows, groups * 4, 32)
    top = v.abs().amax(2)
    bad = ~v.isfinite().all(2)
    exponent = torch.frexp(torch.where(bad | (top == 0), torch.ones_like(top), top)).exponent.double() - 3  # floor(log2) - 2
    exponent = torch.where(top == 0, torch.full_like(exponent, -127.0), exponent.clamp(min=-127.0))
    q = v / torch.exp2(exponent)[..., None]
    q = torch.where(bad[..., None], torch.zeros_like(q), q)
    # nearest level; of two equally near the one of even number
    distance = (q.abs()[..., None] - LEVELS).abs()
    distance[..., 1::2] += 2.0 ** -40  # below any distance that differs from a tie: values have 24 bits
    code = distance.argmin(-1)
    code = torch.where((q.signbit()), code + 8, code)
    scale = torch.where(bad, torch.full_like(exponent, 255.0), exponent + 127)
    return code.view(rows, -1), scale.long()


def layout(code, scale):
    """The bytes of PackedMatrix.codes and .scales."""
    rows = code.shape[0]
    c = code.view(rows, -1, 64, 2).transpose(0, 1)
    return ((c[..., 0] | c[..., 1] << 4).to(torch.uint8).contiguous(),
            scale.view(rows, -1, 4).transpose(0, 1).to(torch.uint8).contiguous())


def values(code, scale, cols):
    """What codes and scales stand for, in 64 bits."""
    rows = code.shape[0]
    v = torch.where(code >= 8, -LEVELS[code & 7], LEVELS[code & 7]).view(rows, -1, 32)
    by = torch.where(scale == 255, torch.full(scale.shape, float("nan"), dtype=torch.float64), torch.exp2(scale.double() - 127))
    return (v * by[..., None]).view(rows, -1)[:, :cols]


def packed_values(x):
    return values(*quantise(x), x.shape[1])


def product(a, b, dtype, old=None):
    """(a b^T, bound): products of codes and scales are exact, k of them and the old
    value are added in binary32 in some order, and the output is rounded once."""
    want, mass = a @ b.t(), a.abs() @ b.abs().t()
    if old is not None:
        want, mass = want + old.double(), mass + old.double().abs()
    u = U[dtype]
    return want, (a.shape[1] + 4) * EPS * mass * (1 + u) + u * want.abs() + TINY[dtype]
