"""Plain 64-bit definitions of the operators around attention, and how far a kernel may be from them.

Tolerances count roundings.  One rounding to a type is off by at most eps / 2 of the value (bf16 2^-8, fp32 2^-24).  An fp32 dot
product of n terms is off by at most (n + 2) 2^-24 of the sum of its terms' magnitudes."""
import math

import numpy as np
import torch

PAGE = 64
U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def starts_of(lens, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def randn(shape, dtype, seed, factor=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * factor).to(dtype)


def strided(x, pad, offset):
    """The same values [tokens, heads, head_dim] with `pad` more elements between tokens, `offset` elements behind an aligned start."""
    n, h, d = x.shape
    pool = torch.full((n * (h * d + pad) + offset,), 3.0, dtype=x.dtype, device=x.device)
    v = pool[offset:].view(n, h * d + pad)[:, :h * d].view(n, h, d) if pad == 0 else pool[offset:].as_strided((n, h, d), (h * d + pad, d, 1), offset)
    v.copy_(x)
    return v


# ---- rotary positions -------------------------------------------------------------------------------


def rope(x, positions, dims, theta, scale, halves, joint, norm, eps):
    """-> (value, tolerance) in 64 bits."""
    x64 = x.double()
    R = sum(dims)
    freq, axis = [], []
    for a, d in enumerate(dims):
        for j in range(d // 2):
            freq.append(scale[a] * (theta[0] ** (-2.0 * len(axis) / R) if joint else theta[a] ** (-2.0 * j / d)))
            axis.append(a)
    angle = positions.double()[:, axis] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    y = x64
    if norm is not None:
        y = x64 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + eps) * norm.double()
    first = torch.arange(R // 2, device="cuda") if halves else torch.arange(0, R, 2, device="cuda")
    second = first + R // 2 if halves else first + 1
    a, b = y[..., first], y[..., second]
    out, size = y.clone(), y.abs()
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    size[..., first] = size[..., second] = a.abs() + b.abs()
    # sum of squares in 18 steps at most, root, quotient, weight; the angle's turn rounded to 2^-25, its sine to a few units; three products
    return out, HALF_STEP[x.dtype] * out.abs() + 32 * U32 * size


# ---- attention --------------------------------------------------------------------------------------


def attention(q, k, v, sees, scale, p_step, dtype):
    """One sequence: q [n, H, hd] over k, v [m, Hkv, hd]; sees [n, m].  p_step: rounding of the probabilities (0: kept in fp32).
    -> (value, tolerance), 0 where nothing is seen."""
    n, H, hd = q.shape
    m, Hkv = k.shape[0], k.shape[1]
    out, tol = torch.zeros((n, H, hd), dtype=torch.float64, device="cuda"), torch.zeros((n, H, hd), dtype=torch.float64, device="cuda")
    if m == 0 or n == 0:
        return out, tol
    some = sees.any(1)
    for h in range(H):
        a, b, w = q[:, h].double(), k[:, h // (H // Hkv)].double(), v[:, h // (H // Hkv)].double()
        s = torch.where(sees, a @ b.T.contiguous() * scale, -math.inf)
        # magnitude of the terms of the scores that count, for the error of a score
        mag = torch.where(sees, a.abs() @ b.abs().T.contiguous() * scale, 0.0).amax(1)
        p = torch.exp(s - s.amax(1, keepdim=True))
        p = torch.where(some[:, None], p / p.sum(1, keepdim=True), 0.0)
        o, size = p @ w, p @ w.abs()
        out[:, h] = o
        err = 2 * (hd + 6) * U32 * mag + (m + 32) * U32
        tol[:, h] = HALF_STEP[dtype] * o.abs() + (p_step + err[:, None]) * (1 + HALF_STEP[dtype]) * size
    return torch.where(some[:, None, None], out, 0.0), torch.where(some[:, None, None], tol, 0.0)


def close(got, value, tol, what=""):
    off = (got.double() - value).abs() - tol
    bad = ~(off <= 0)
    assert not bad.any(), (what, int(bad.sum()), float(off[bad].nan_to_num(nan=math.inf).max()), bad.nonzero()[:4].tolist())


# ---- the cache --------------------------------------------------------------------------------------


def codes():
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = math.nan if (b & 127) == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = -x if b & 128 else x
    return out


CODES = codes()
FINITE = np.sort(CODES[:127])


def encode(x):
    """Nearest e4m3 code of scaled values (float64 array), ties to even, saturating, NaN to NaN."""
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(FINITE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - FINITE[lo], FINITE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(FINITE[hi] == a, hi, code)
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


PLACE = np.array([16 * (t % 16 // 4) + 4 * (t // 16) + t % 4 for t in range(PAGE)])


class Cache:
    """The cache in 64 bits: bytes by token [pages, heads, 64, hd] and scales, for k and for v."""

    def __init__(self, dev):
        self.b = [dev.k.cpu().numpy().copy(), dev.v.cpu().numpy().transpose(0, 1, 3, 2)[:, :, PLACE].copy()]
        self.s = [dev.k_scale.cpu().numpy().astype(np.float64).copy(), dev.v_scale.cpu().numpy().astype(np.float64).copy()]

    def store(self, table, past, k, v, starts, lens):
        pages = self.b[0].shape[0]
        for which, x in enumerate((k.double().cpu().numpy(), v.double().cpu().numpy())):
            for s, n in enumerate(lens):
                run = x[starts[s]:starts[s] + n]
                for j in range(past[s] // PAGE, (past[s] + n - 1) // PAGE + 1 if n else 0):
                    page = table[s][j] if j < len(table[s]) else -1
                    lo, hi = max(0, past[s] - j * PAGE), min(PAGE, past[s] + n - j * PAGE)
                    new = run[j * PAGE + lo - past[s]:j * PAGE + hi - past[s]]
                    if not 0 <= page < pages:
                        continue
                    for h in range(new.shape[1]):
                        f = np.abs(new[:, h])
                        top = f[np.isfinite(f)].max(initial=0.0)
                        e = -100
                        while e < 119 and top > 448.0 * 2.0 ** e:
                            e += 1
                        sc = 2.0 ** e
                        if lo:
                            sc = max(sc, self.s[which][page, h])
                        old = CODES[self.b[which][page, h, :lo]] * (self.s[which][page, h] / sc)
                        self.b[which][page, h] = 0
                        self.b[which][page, h, :lo] = encode(old)
                        self.b[which][page, h, lo:hi] = encode(new[:, h] / sc)
                        self.s[which][page, h] = sc

    def values(self, which, table_row, tokens):
        """[tokens, heads, hd] in 64 bits on the device, and which of the tokens are held."""
        pages, H, _, hd = self.b[which].shape
        out, held = np.zeros((tokens, H, hd)), np.zeros(tokens, bool)
        for j in range((tokens + PAGE - 1) // PAGE):
            p = table_row[j] if j < len(table_row) else -1
            if 0 <= p < pages:
                n = min(PAGE, tokens - j * PAGE)
                out[j * PAGE:j * PAGE + n] = (CODES[self.b[which][p]] * self.s[which][p][:, None, None]).transpose(1, 0, 2)[:n]
                held[j * PAGE:j * PAGE + n] = True
        return torch.from_numpy(out).cuda(), torch.from_numpy(held).cuda()
