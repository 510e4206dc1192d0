"""Plain forms of the serving operators in 64 bits (torch on the CPU), and the inputs of their tests."""
import math

import torch

F64 = torch.float64


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, seed, std=1.0):
    return torch.randn(shape, generator=gen(seed), dtype=torch.float32) * std


# ------------------------------------------------------------------------------------------- norm --

def rmsnorm(x, residual, weight, eps):
    """h and y."""
    h = x.to(F64) + (residual.to(F64) if residual is not None else 0)
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, h * r * weight.to(F64), r


def rmsnorm_codes(x, residual, weight):
    """Codes and steps (before the factor r), in fp32 with one rounding a line as the interface says."""
    h = x.float() + (residual.float() if residual is not None else 0)
    return codes_of(h * weight.float())


def codes_of(u):
    """Signed codes of fp32 rows and their step max / 127."""
    most = u.abs().amax(-1)
    step = torch.where(most > 0, most / torch.tensor(127.0), torch.tensor(1.0))
    return (u / step[..., None]).round().clamp(-127, 127).to(torch.int8), step


def rmsnorm_backward(h, weight, eps, dy, dres):
    """dx, dweight and the magnitudes that their rounding errors go by."""
    h, w, dy = h.to(F64), weight.to(F64), dy.to(F64)
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    n, g = h * r, dy * w
    mean = (g * n).mean(1, keepdim=True)
    dx = r * (g - n * mean)
    size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    if dres is not None:
        dx, size = dx + dres.to(F64), size + dres.to(F64).abs()
    return dx, size, (dy * n).sum(0), (dy * n).abs().sum(0)


# ------------------------------------------------------------------------------- cache and attention --

class Step:
    """A cache, requests and new tokens: `new` and `lens` are lists (lens with the new tokens).  Slots that no token lies in hold NaN (their
    steps, in a cache of bytes), entries of the page table that no token lies in hold numbers that are no page."""

    def __init__(self, new, lens, heads, kv_heads, dim, page, eight, seed, spare=3, pad=0, pool=None):
        self.new, self.lens, self.heads, self.kv_heads, self.dim, self.page, self.eight = new, lens, heads, kv_heads, dim, page, eight
        self.tokens = sum(new)
        pages = [-(-max(n, 0) // page) for n in lens]
        self.max_pages = max(max(pages), 1) + 1
        count = pool or sum(pages) + spare
        order = torch.randperm(count, generator=gen(seed))[:sum(pages)].tolist() if pool is None else list(range(count - sum(pages), count))
        self.table = torch.full((len(new), self.max_pages), -7, dtype=torch.int32)
        self.table[:, -1] = 2 ** 31 - 1
        for r, n in enumerate(pages):
            self.table[r, :n] = torch.tensor(order[:n], dtype=torch.int32)
            order = order[n:]
        self.num_pages = count
        self.starts = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32)
        self.kv_len = torch.tensor(lens, dtype=torch.int32)
        wide = (heads + 2 * kv_heads) * dim + pad     # the new tokens as a fused linear writes them, `pad` more columns
        self.qkv = normal((max(self.tokens, 1), wide), seed + 1).to(torch.bfloat16)
        # the values that the requests' tokens stand for, in 64 bits, [kv_heads, len, dim]
        self.values = []
        for r, n in enumerate(lens):
            kv = []
            for i in range(2):
                t = normal((kv_heads, max(n, 0), dim), seed + 10 + 2 * r + i)
                kv.append(codes_of(t) if eight else t.to(torch.bfloat16))
            self.values.append(kv)

    def split(self, t):
        a, b = self.heads * self.dim, self.kv_heads * self.dim
        cut = lambda i, n: t[:self.tokens, i:i + n].unflatten(1, (n // self.dim, self.dim))  # noqa: E731
        return cut(0, a), cut(a, b), cut(a + b, b)

    def pools(self, device):
        """k, v, k_scale, v_scale on the device, filled."""
        shape = (self.num_pages, self.kv_heads, self.page, self.dim)
        out, scales = [], []
        for i in range(2):
            if self.eight:
                data = torch.full(shape, -128, dtype=torch.int8, device=device)
                scale = torch.full(shape[:3], math.nan, device=device)
            else:
                data, scale = torch.full(shape, math.nan, dtype=torch.bfloat16, device=device), None
            for r, n in enumerate(self.lens):
                for p in range(-(-max(n, 0) // self.page)):
                    lo, hi, at = p * self.page, min(n, (p + 1) * self.page), int(self.table[r, p])
                    if self.eight:
                        codes, step = self.values[r][i]
                        data[at, :, :hi - lo] = codes[:, lo:hi].to(device)
                        scale[at, :, :hi - lo] = step[:, lo:hi].to(device)
                    else:
                        data[at, :, :hi - lo] = self.values[r][i][:, lo:hi].to(device)
            out.append(data)
            scales.append(scale)
        return out[0], out[1], scales[0], scales[1]

    def real(self, r, i):
        v = self.values[r][i]
        return v[0].to(F64) * v[1].to(F64)[..., None] if self.eight else v.to(F64)


def attend(s, scale):
    """Outputs [tokens, heads, dim] in 64 bits, and the bound of the kernel's error: p rounded to bf16 (2^-8 of it), scores off by the fp32
    rounding of dim products (each side of the quotient), the exponential and the sums (2^-18), the output rounded to bf16; a p below
    the smallest normal number, 2^-126, may count as zero."""
    q = s.split(s.qkv)[0].to(F64)
    out = torch.zeros((s.tokens, s.heads, s.dim), dtype=F64)
    tol = torch.zeros_like(out)
    group = s.heads // s.kv_heads
    for r, (n, length) in enumerate(zip(s.new, s.lens)):
        if n == 0 or length <= 0:
            continue
        t0 = int(s.starts[r])
        k, v = s.real(r, 0), s.real(r, 1)
        pos = torch.arange(length - n, length)[:, None]
        seen = torch.arange(length)[None] <= pos
        for h in range(s.heads):
            x = q[t0:t0 + n, h]
            sc = (x @ k[h // group].T) * scale
            size = (x.abs() @ k[h // group].abs().T * scale).masked_fill(~seen, 0).amax(1)
            sc = sc.masked_fill(~seen, -math.inf)
            top = sc.amax(1, keepdim=True).clamp(min=-1e300)
            e = torch.exp(sc - top)
            total = e.sum(1, keepdim=True)
            p = e / torch.where(total > 0, total, 1.0)
            o = p @ v[h // group]
            spread = p @ v[h // group].abs()
            out[t0:t0 + n, h] = o
            tol[t0:t0 + n, h] = 2 ** -8 * o.abs() + (2 ** -8 + 2 * (s.dim + 8) * 2 ** -24 * size[:, None] + 2 ** -18) * spread + 2 ** -126 * v[h // group].abs().sum(0)
    return out, tol


def angles(positions, dim, seed=None):
    at = torch.arange(positions, dtype=F64)[:, None]
    a = at * 10000.0 ** (-torch.arange(dim // 2, dtype=F64) * 2 / dim)
    return a.cos().float(), a.sin().float()


def rotate(t, cos, sin):
    """fp32, each product and sum rounded once."""
    half = t.shape[-1] // 2
    a, b = t[..., :half], t[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def positions(s):
    """(request, position) of each new token."""
    return [(r, length - n + i) for r, (n, length) in enumerate(zip(s.new, s.lens)) for i in range(n)]
