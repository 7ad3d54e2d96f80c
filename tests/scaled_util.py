"""Plain models (64 bits, Python loops) of the rotation and of a cache of e4m3 codes with scales."""
import numpy as np
import torch

import paged_util as plain

F8 = torch.float8_e4m3fn


def turn(x, pos, freq, interleaved, amplitude=1.0):
    """x [B,N,H,D] (float64 array) rotated; pos [B,N], freq float32 [F]."""
    y, F = x.copy(), len(freq)
    t = pos.astype(np.float64)[:, :, None, None] * freq.astype(np.float64)
    c, s = amplitude * np.cos(t), amplitude * np.sin(t)
    one, two = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if interleaved else (slice(0, F), slice(F, 2 * F))
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    return y


def encode(values):
    """float64 -> codes (uint8); what is not finite, NaN."""
    v = torch.from_numpy(np.where(np.isfinite(values), values, np.nan)).float().clamp(-448, 448)
    return v.to(F8).view(torch.uint8).numpy()


def decode(codes):
    return torch.from_numpy(np.ascontiguousarray(codes)).view(F8).double().numpy()


def fitting(most):
    s = 2.0 ** -60
    while s < 2.0 ** 60 and not most <= 448 * s:
        s *= 2
    return s


def limited(s):
    return 2.0 ** -60 if np.isnan(s) else min(max(float(s), 2.0 ** -60), 2.0 ** 60)


def write(codes, scales, table, kv_len, values, counts):
    """values float64 [B,N,H_kv,D], rows i < counts[b]; codes uint8 [P,H_kv,page,D], scales float32."""
    P, H, page, _ = codes.shape
    for b in range(values.shape[0]):
        L, n = int(kv_len[b]), int(counts[b])
        if L < 0:
            continue
        for first in range(L // 16 * 16, L + n, 16):
            at = plain.row_of(table, page, P, b, first)
            if at is None:
                continue
            p, r = at
            lo, hi = max(L - first, 0), min(L + n - first, 16)
            for h in range(H):
                v = values[b, first + lo - L:first + hi - L, h]
                s = fitting(np.abs(v[np.isfinite(v)]).max(initial=0.0))
                if lo > 0:
                    old = limited(scales[p, h, r // 16])
                    s = max(s, old)
                    if s != old:
                        codes[p, h, r:r + lo] = encode(decode(codes[p, h, r:r + lo]) * (old / s))
                codes[p, h, r + lo:r + hi] = encode(v / s)
                scales[p, h, r // 16] = s


def commit(codes, scales, table, kv_len, nodes, lens, N):
    P, H, page, D = codes.shape
    B, depth = nodes.shape
    held, counts = np.zeros((B, depth, H, D)), np.zeros(B, int)
    for b in range(B):
        counts[b] = min(max(int(lens[b]), 0), depth)
        for i in range(counts[b]):
            at = plain.row_of(table, page, P, b, int(kv_len[b]) + min(max(int(nodes[b, i]), 0), N - 1))
            if at:
                p, r = at
                held[b, i] = decode(codes[p, :, r]) * np.array([limited(s) for s in scales[p, :, r // 16]])[:, None]
    write(codes, scales, table, kv_len, held, counts)


def same_codes(got, want):
    """Codes as a tensor against an array: equal values, all NaN alike."""
    g, w = decode(got.view(torch.uint8).cpu().numpy()), decode(want)
    return np.array_equal(g, w, equal_nan=True)


def pool(rng, P, H, page, D, layout="hnd"):
    """Codes (finite) and scales of a pool on the GPU, K and V, and the same as arrays."""
    raw = rng.integers(0, 256, (2, P, H, page, D), dtype=np.uint8)
    raw[(raw & 127) == 127] = 0
    scales = 2.0 ** rng.integers(-9, -4, (2, P, H, page // 16)).astype(np.float32)
    t = torch.from_numpy(raw).cuda()
    if layout == "nhd":
        t = t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    elif layout == "gap":                               # K and V interleaved in one allocation
        t = t.transpose(0, 1).contiguous().transpose(0, 1)
    s = torch.from_numpy(scales).cuda()
    return t[0].view(F8), t[1].view(F8), s[0], s[1], raw.copy(), scales.copy()


def tables(rng, B, W, P):
    return rng.permutation(P)[:B * W].reshape(B, W).astype(np.int32)
