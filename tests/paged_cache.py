"""A model of the paged cache in 64 bits, place by place: rotation, the 4-bit groups, where an octet keeps what, attention over it."""
import numpy as np
import torch


def rotated(x, positions, freq, interleaved):
    """[T, heads, dim] float64; angles, cosines, sines and sums in 64 bits."""
    y = x.copy()
    half = 0 if freq is None else len(freq)
    for c in range(half):
        a, b = (2 * c, 2 * c + 1) if interleaved else (c, c + half)
        angle = (positions.astype(np.float64) * freq[c])[:, None]
        y[:, :, a] = x[:, :, a] * np.cos(angle) - x[:, :, b] * np.sin(angle)
        y[:, :, b] = x[:, :, b] * np.cos(angle) + x[:, :, a] * np.sin(angle)
    return y


def rotated32(x, positions, freq, interleaved):
    """The same as documented: cosines and sines rounded to 32 bits, products and sums one by one."""
    y = x.astype(np.float32)
    half = 0 if freq is None else len(freq)
    for c in range(half):
        a, b = (2 * c, 2 * c + 1) if interleaved else (c, c + half)
        angle = (positions.astype(np.float64) * freq[c])[:, None]
        cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        xa, xb = x[:, :, a].astype(np.float32), x[:, :, b].astype(np.float32)
        y[:, :, a] = xa * cos - xb * sin
        y[:, :, b] = xb * cos + xa * sin
    return y


def groups(x):
    """Codes (0 .. 15) and fp16 scales of [..., dim] float32, and the quotients x / s in 64 bits."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    hi, lo = x.max(-1), x.min(-1)
    peak = np.where(hi >= -lo, hi, lo)
    scale = np.clip(peak.astype(np.float64) / -8, -65504, 65504).astype(np.float16)
    s = scale.astype(np.float64)[..., None]
    quotient = np.divide(x.astype(np.float64), s, out=np.zeros(x.shape), where=s != 0)
    code = np.clip(np.rint(quotient), -8, 7) + 8
    return code.astype(np.uint8), scale, quotient


def places(dim):
    """Of (token, dim) in an octet: byte and shift of the code and index of the 16-bit scale, for keys and for values."""
    J, at = dim // 32, {}
    for t in range(8):
        for d in range(dim):
            j, r = divmod(d, 32)
            at[0, t, d] = (t * (dim // 2) + ((r // 8) * J + j) * 4 + (r % 8) // 2, 4 * (d % 2), 2 * dim + t * J + j)
            half = ((r // 4) * 4 + t // 2) * J * 2 + j * 2 + t % 2
            at[1, t, d] = (4 * dim + dim // 2 + 2 * half + (r % 4) // 2, 4 * (d % 2), (8 * dim + dim // 2) // 2 + (t // 2) * J * 2 + j * 2 + t % 2)
    return at


def tables(dim):
    """The same as arrays [2, 8, dim]: byte, shift, scale."""
    at = places(dim)
    out = np.zeros((3, 2, 8, dim), dtype=np.int64)
    for (kind, t, d), v in at.items():
        out[:, kind, t, d] = v
    return out


def write4(data, block_size, slot, k, v):
    """Puts one token's keys and values [heads, dim] float32 into data [blocks, heads, block / 8, 9 dim] uint8."""
    dim = k.shape[-1]
    byte, shift, word = tables(dim)
    block, at = divmod(int(slot), block_size)
    for h in range(k.shape[0]):
        octet = data[block, h, at // 8]
        scales = octet.view(np.float16)
        for kind, x in enumerate((k[h], v[h])):
            code, scale, _ = groups(x[None])
            scales[word[kind, at % 8]] = scale.repeat(32, -1)[0]
            for d in range(dim):
                p, z = byte[kind, at % 8, d], shift[kind, at % 8, d]
                octet[p] = (octet[p] & ~np.uint8(15 << z)) | (code.reshape(-1)[d] << z)


def read4(data, block_size, slots):
    """keys, values [T, heads, dim] float64 of the slots (zeros where there is none)."""
    N, H, _, size = data.shape
    dim = size // 9
    byte, shift, word = tables(dim)
    out = np.zeros((2, len(slots), H, dim))
    for i, slot in enumerate(slots):
        if not 0 <= slot < N * block_size:
            continue
        block, at = divmod(int(slot), block_size)
        octet = data[block, :, at // 8]
        scales = np.ascontiguousarray(octet).view(np.float16).astype(np.float64)
        for kind in range(2):
            code = (octet[:, byte[kind, at % 8]] >> shift[kind, at % 8]) & 15
            out[kind, i] = (code.astype(np.float64) - 8) * scales[:, word[kind, at % 8]]
    return out[0], out[1]


def to_numpy(t):
    """A tensor's numbers (16-bit types as float32)."""
    return t.detach().float().cpu().numpy() if t.dtype in (torch.bfloat16, torch.float16) else t.detach().cpu().numpy()


def cast(x, dtype):
    """float64 numbers rounded to a torch type, as float64."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).double().numpy()


def all4(data):
    """(keys, values, their scales) [slots, heads, dim] float64 of a whole cache [blocks, heads, block / 8, 9 dim] uint8."""
    N, H, O, size = data.shape
    dim = size // 9
    byte, shift, word = tables(dim)
    scales = np.ascontiguousarray(data).view(np.float16).astype(np.float64)
    out = []
    for kind in range(2):
        code = (data[..., byte[kind]] >> shift[kind]) & 15
        s = scales[..., word[kind]]
        out += [(code.astype(np.float64) - 8) * s, s]
    k, ks, v, vs = (x.transpose(0, 2, 3, 1, 4).reshape(N * O * 8, H, dim) for x in out)
    return k, v, ks, vs


def attention(q, held, block_size, table, offsets, positions, scale, window):
    """What gr_cache_attend computes, in 64 bits, and a bound of its error before the rounding to the output's type.

    x = scale q.k is summed in 32 bits, from codes 0 .. 15 and the sum of the queries times 8, both up to A = scale sum |q| 16 |s|: eight
    roundings of 2^-23 A.  p is rounded to 11 bits and p s once more, 2^-12 of each, and what comes of it is taken u - 8 times, 8 at most: 16 2^-12 p |s|.
    Where they are below 2^-14 they are off by 2^-25 each instead, of a reference up to 2^4 above the largest p: by 2^-21 of that, (1 + |s|) 8 times.
    Sums of n / 16 products and eight joins round 2^-22 of 16 p |s| each."""
    T, Hq, D = q.shape
    k, v, ks, vs = held
    H = k.shape[1]
    out, bound = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for r in range(len(offsets) - 1):
        for i in range(offsets[r], offsets[r + 1]):
            p0 = int(positions[offsets[r]])
            p = p0 + i - int(offsets[r])
            if p0 < 0:
                continue
            t = np.arange(max(0, p - window + 1) if window else 0, min(p + 1, table.shape[1] * block_size))
            block = table[r, t // block_size]
            t = t[(block >= 0) & (block * block_size < len(k))]
            z = table[r, t // block_size] * block_size + t % block_size
            if not len(z):
                continue
            for h in range(Hq):
                g = h // (Hq // H)
                x = scale * (k[z, g] @ q[i, h])
                dx = 8 * 2.0 ** -23 * (abs(scale) * 16 * np.abs(ks[z, g]) @ np.abs(q[i, h])).max()
                w = np.exp(x - x.max())
                out[i, h] = w @ v[z, g] / w.sum()
                s = np.abs(vs[z, g])
                bound[i, h] = ((16 * 2.0 ** -12 + 16 * (len(z) / 16 + 8) * 2.0 ** -22) * (w @ s) + 2.0 ** -21 * 8 * (1 + s).sum(0)
                               + (2 * dx + 2.0 ** -20) * (w @ np.abs(v[z, g]))) / w.sum()
    return out, bound
