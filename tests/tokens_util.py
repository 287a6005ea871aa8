"""Plain 64-bit forms of the calls on several new tokens per sequence, and the caches that their tests use."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
WIDE = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.bfloat16}
# half a step of a rounding to the type, relative to the value
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4}


def descriptor(rkv, batch, hkv, hq, d, dtype, status, table=None, pages=0):
    x = rkv.rkv_desc_default()
    x.batch, x.n_kv_heads, x.n_q_heads, x.head_dim = batch, hkv, hq, d
    x.dtype = {"bf16": rkv.RKV_BF16, "f32": rkv.RKV_F32, "fp8": rkv.RKV_FP8_E4M3}[dtype]
    x.device_status = status.data_ptr()
    if table is not None:
        x.block_table, x.pool_pages = table.data_ptr(), pages
    return x


def random_rows(shape, dtype, gen, nan_from=None):
    """Values of a cache type; rows from nan_from[b] on are NaN (nothing may come from there)."""
    x = torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype])
    if nan_from is not None:
        for b, n in enumerate(nan_from):
            x.view(torch.uint8).view(shape[0], shape[1], shape[2], -1)[b, :, max(n, 0):] = 0x7F if dtype == "fp8" else 0xFF
    return x


def to_pages(x, gen, spare=3):
    """[batch, hkv, cap, d] -> (pool of pages in random order with NaN pages in between, table, pages)."""
    b, h, cap, d = x.shape
    need = b * h * cap // 128
    order = torch.randperm(need + spare, generator=gen, device="cuda")[:need]
    pool = torch.empty(need + spare, 128, d, dtype=x.dtype, device="cuda")
    raw = pool.view(torch.uint8)
    raw.fill_(0x7F if x.dtype == torch.float8_e4m3fn else 0xFF)
    raw[order] = x.contiguous().view(torch.uint8).view(need, 128, -1)
    return pool, order.view(b, h, cap // 128).to(torch.int32).contiguous()


def from_pages(pool, table, d):
    b, h, n = table.shape
    return pool.view(torch.uint8)[table.flatten().long()].view(pool.dtype).view(b, h, n * 128, d)


def rotation_table(rows, dim, base=10000.0):
    angle = np.arange(rows, dtype=np.float64)[:, None] * base ** (-2.0 * np.arange(dim // 2) / dim)
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()


def rotate(x, pos, dim, interleaved, base=10000.0):
    """x [n, heads, d] in 64 bits by complex products; also |x| + |y| of every element's pair (0 where nothing turns)."""
    y, size = x.clone(), torch.zeros_like(x)
    if dim:
        i = torch.arange(dim // 2, device=x.device)
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)
        angle = pos.double()[:, None] * base ** (-2.0 * i.double() / dim)
        z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        y[..., lo], y[..., hi] = z.real, z.imag
        size[..., lo] = size[..., hi] = x[..., lo].abs() + x[..., hi].abs()
    return y, size


def rounding_tolerance(ref, size, dtype):
    """Half a step of the one rounding to `dtype`, and before it: cosine, sine, two products and a sum of fp32, each off by at most
    2^-24 of a product, in all below 2^-21 of |x| + |y|.  E4M3 values under 2^-6 have steps of 2^-9, half of which is 2^-10."""
    tol = ref.abs() * HALF_STEP[dtype] + size * 2.0 ** -21
    return tol + (2.0 ** -10 if dtype == torch.float8_e4m3fn else 0.0)


def attention(q, keys, values, visible):
    """q [n, G, d], keys and values [rows, d], visible [n, rows]: softmax(q k / sqrt(d)) v in 64 bits, zeros where nothing is visible;
    also the weighted mean of |v|, which bounds what errors of the weights can do."""
    q, keys, values = q.double(), keys.double(), values.double()
    x = torch.einsum("ngd,jd->ngj", q, keys) / q.shape[-1] ** 0.5
    x = x.masked_fill(~visible[:, None], -float("inf"))
    top = x.amax(-1, keepdim=True)
    w = torch.where(visible[:, None], (x - torch.where(top.isinf(), 0.0, top)).exp(), 0.0)
    total = w.sum(-1, keepdim=True)
    w = torch.where(total > 0, w / total.clamp_min(1e-300), 0.0)
    return torch.einsum("ngj,jd->ngd", w, values), torch.einsum("ngj,jd->ngd", w, values.abs())


def attention_tolerance(ref, size, rows, d, out_type):
    """Values N(0, 1).  A score's products are added up in fp32: off by at most (d + 2) 2^-24 sum |q k| / sqrt(d), and sum |q k| <= |q| |k|
    < 2 d; the exponential adds 2^-20.  Such an error of every weight moves the result by twice it, relative to the weighted mean of |v|
    (numerator and denominator); adding up `rows` weighted values adds rows 2^-24.  bf16 products round the weights (half a step of
    bf16).  Then one rounding to the output's type."""
    delta = (d + 2) * 2.0 ** -24 * 2 * d ** 0.5 + 2.0 ** -20
    weights = 2.0 ** -8 if out_type == torch.bfloat16 else 0.0
    inner = size * (2 * delta + rows * 2.0 ** -24 + weights)
    return inner + (ref.abs() + inner) * HALF_STEP[out_type]
