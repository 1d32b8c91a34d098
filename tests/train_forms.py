"""What the tests of the training calls share: routings and where their rows lie, and the layer's definitions in 64 bits on the CPU."""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def dtype_of(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def routing(gen, T, E, k, capacity=0, skew=1.0):
    """topk_idx [T,k], inv_perm [T*k] and counts [E] (int32, on the CPU) of a skewed random gate; slots an expert has no room for: -1."""
    idx = torch.topk(torch.randn(T, E, generator=gen) + skew * torch.randn(E, generator=gen), k, dim=1).indices
    flat = idx.reshape(-1)
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k)
    counts = torch.bincount(flat, minlength=E)
    if capacity:
        rank = place - (torch.cumsum(counts, 0) - counts)[flat]
        place = torch.where(rank < capacity, flat * capacity + rank, -1)
    return idx.to(torch.int32), place.to(torch.int32), counts.to(torch.int32)


def weights(gen, T, k):
    return torch.softmax(torch.randn(T, k, generator=gen), 1)


def used_rows(counts, capacity):
    return (torch.arange(capacity)[None, :] < counts[:, None].long()).reshape(-1)


def encode(x):
    """[n, f] fp64 -> the values of the codes and the exponents (+127) of the blocks of 32; values that are not finite: NaN codes."""
    f = x.shape[1]
    blocks = -(-f // 32)
    finite = torch.isfinite(x)
    padded = torch.zeros(x.shape[0], blocks * 32, dtype=torch.float64)
    padded[:, :f] = torch.where(finite, x, 0.0)
    most = padded.reshape(-1, blocks, 32).abs().amax(-1)
    byte = torch.zeros(most.shape, dtype=torch.int64)
    for e in range(-127, 128):  # the least power of two that brings the largest to 448
        byte[most > 448.0 * 2.0 ** e] = e + 128
    v = torch.where(finite, x, 0.0) / torch.exp2(byte.double() - 127.0).repeat_interleave(32, 1)[:, :f]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.where(finite, torch.round(v / step) * step, float("nan")), byte


def code_values(codes):
    return codes.view(torch.float8_e4m3fn).float().double()


def decode(codes, scales):
    """codes [n, 2, f], scales [n, 2, blocks] bytes -> g, u in fp64."""
    v = code_values(codes) * torch.exp2(scales.double() - 127.0).repeat_interleave(32, 2)[:, :, :codes.shape[2]]
    return v[:, 0], v[:, 1]
