"""The rule of 8-bit checkpoints for whole matrices at a time (ref_layers.pack takes them value by value), in 64 bits on the CPU."""
import torch

from tests import ref_layers as ref


def pack(x):
    """(codes, exponent bytes, values), as ref_layers.pack returns them."""
    top = 10 if x.dtype == torch.float16 else 122
    n, d = x.shape
    groups = -(-d // ref.GROUP)
    v = torch.nn.functional.pad(x.detach().cpu().double(), (0, groups * ref.GROUP - d)).view(n, groups, ref.GROUP)
    fine = torch.isfinite(v).all(2)
    v = torch.where(fine.unsqueeze(2), v, 0.0)
    largest = v.abs().amax(2)
    # largest = m * 2^k, 1/2 <= m < 1: 127 * 2^(k-7) or 127 * 2^(k-6) is the least that holds it
    m, k = torch.frexp(largest)
    e = torch.where(m > 127 / 128, k - 6, k - 7).clamp(min=-130)
    e = torch.where(largest == 0, -130, e).double()
    limit = torch.where(e == top, 63.0, 127.0).unsqueeze(2)
    q = (v / torch.exp2(e).unsqueeze(2)).round()
    q = torch.maximum(torch.minimum(q, limit), -limit)
    values = torch.where(fine.unsqueeze(2), q * torch.exp2(e).unsqueeze(2), float("nan"))
    bytes_ = torch.where(fine, e + 130, 255.0).to(torch.uint8)
    return q.flatten(1)[:, :d].to(torch.int8).contiguous(), bytes_, values.flatten(1)[:, :d].contiguous()
