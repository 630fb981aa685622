"""Plain 64-bit statements of the calls for 8-bit layers and of what stands around a layer, and buffers with a rim."""
import math

import torch

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS32 = 2.0 ** -24                                        # half a unit of binary32
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": EPS32}  # half a unit in the last place of a value, relative
LEAST = {"f16": 2.0 ** -25, "bf16": 0.0, "f32": 0.0}      # the same of fp16's smallest values


class Rim:
    """A matrix of `rows` x `n` values inside a buffer that is set to `fill` all around: rows `ld` apart, `lead` values in
    front of the first."""

    def __init__(self, rows, n, dtype, ld=None, lead=0, fill=None):
        self.rows, self.n, self.ld, self.lead = rows, n, n if ld is None else ld, lead
        self.fill = fill if fill is not None else 77
        self.flat = torch.full((lead + rows * self.ld + 64,), self.fill, dtype=dtype, device="cuda")
        self.view = self.flat[lead:lead + rows * self.ld].view(rows, self.ld)[:, :n]
        self.pointer = self.flat.data_ptr() + lead * self.flat.element_size()

    def set(self, values):
        self.view.copy_(values)
        return self

    def rim_is_whole(self):
        seen = self.flat.clone()
        seen[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.n] = self.fill
        return bool((seen == self.fill).all())


def hadamard(block):
    H = torch.ones(1, 1, dtype=torch.float64)
    while H.shape[0] < block:
        H = torch.cat((torch.cat((H, H), 1), torch.cat((H, -H), 1)), 0)
    return H.cuda()


def rotate(v, signs, block):
    v = v * signs.double()
    return (v.reshape(-1, block) @ hadamard(block)).reshape(v.shape) / math.sqrt(block)


def silu(v):
    return v / (1 + torch.exp(-v))


def normed(v, layer, eps, weight, bias):
    if layer:
        v = v - v.mean(dim=1, keepdim=True)
    v = v / (v.square().mean(dim=1, keepdim=True) + eps).sqrt() * weight.double()
    return v if bias is None else v + bias.double()


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def signs_of(g, n):
    return (torch.randint(0, 2, (n,), device="cuda", generator=g) * 2 - 1).to(torch.int8)
