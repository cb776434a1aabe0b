"""A plain fp64 model of the 8-bit cache and of the attentions over it, for the tests:
numpy only, written from the definitions (see jl_cache8 in include/jetlong.h)."""
import math

import numpy as np

D = 128
BLOCK = 64
E_MIN, E_MAX = -117, 119
U16, UBF = 2.0 ** -11, 2.0 ** -8  # half a step of fp16 and of bf16, relative to the value


def _table():
    """The 256 numbers of OCP e4m3 (no infinity; 0x7f and 0xff are NaN)."""
    t = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if (b & 127) == 127:
            x = math.nan
        t[b] = -x if b & 128 else x
    return t


E4M3 = _table()


def e4m3(x):
    """fp64 values -> e4m3 bytes: nearest, ties to even, saturating, NaN kept (its sign is free)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    e = np.maximum(np.frexp(np.where(np.isnan(a), 1.0, a))[1] - 1, -6)
    n = np.where(np.isnan(a), 0, np.round(np.where(np.isnan(a), 0, a) / 2.0 ** (e - 3)))  # half to even
    up = n == 16  # rounded to the next power of two
    e, n = np.where(up, e + 1, e), np.where(up, 8, n)
    byte = np.where(n < 8, n, (e + 7) * 8 + (n - 8)).astype(np.int64)
    byte = np.where(np.isnan(x), 127, byte)
    return (byte | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(top):
    """2^e for the smallest e in [E_MIN, E_MAX] with top <= 448 * 2^e."""
    e = np.full(np.shape(top), E_MIN)
    for k in range(E_MIN, E_MAX):
        e = np.where(np.asarray(top) > 448.0 * 2.0 ** k, k + 1, e)
    return 2.0 ** e.astype(np.float64)


def pack_k(y):
    """bytes [..., 64, 128] -> K image [..., 8192]"""
    out = np.zeros(y.shape[:-2] + (BLOCK * D,), dtype=y.dtype)
    for key in range(BLOCK):
        a, t, r = key >> 5, (key >> 4) & 1, key & 15
        d = np.arange(D)
        p, u, g, j = d >> 6, (d >> 5) & 1, (d >> 3) & 3, d & 7
        out[..., ((((a * 2 + t) * 2 + u) * 4 + g) * 16 + r) * 16 + 2 * j + p] = y[..., key, :]
    return out


def pack_v(y):
    out = np.zeros(y.shape[:-2] + (BLOCK * D,), dtype=y.dtype)
    for key in range(BLOCK):
        a, t, g, i = key >> 5, (key >> 4) & 1, (key >> 2) & 3, key & 3
        d = np.arange(D)
        c, e, m = d >> 5, (d >> 4) & 1, d & 15
        out[..., (((a * 4 + c) * 4 + g) * 16 + m) * 16 + 8 * e + 4 * t + i] = y[..., key, :]
    return out


def to_bf16(x):
    """fp64 -> the nearest bf16 as fp64 (through fp32 rounded to odd: one rounding)."""
    x = np.asarray(x, dtype=np.float64)
    f = x.astype(np.float32)
    b = f.view(np.uint32).copy()
    over = np.abs(f.astype(np.float64)) > np.abs(x)
    b = np.where(over, b - 1, b)  # toward zero
    inexact = b.view(np.float32).astype(np.float64) != x
    b = np.where(inexact & ~np.isnan(x), b | 1, b)
    r = ((b.astype(np.uint64) + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    return r.view(np.float32).astype(np.float64)


class Model:
    """A cache by its logical rows: bytes [B, n_blocks, Hkv, 64, 128], scales, means."""

    def __init__(self, B, n_blocks, Hkv):
        self.B, self.nb, self.Hkv = B, n_blocks, Hkv
        self.k = np.zeros((B, n_blocks, Hkv, BLOCK, D), dtype=np.uint8)
        self.v = np.zeros_like(self.k)
        self.ks = np.zeros((B, n_blocks, Hkv))
        self.vs = np.zeros_like(self.ks)
        self.mean = np.zeros((B, n_blocks, Hkv, D))
        self.touched = np.zeros((B, n_blocks), dtype=bool)

    def append(self, k, v, starts, n_new=None, dropped=()):
        """k, v fp64 [B, n, Hkv, 128]; dropped: (b, block) whose page is outside the pool."""
        n = k.shape[1]
        cap = self.nb * BLOCK
        for b in range(self.B):
            m = n if n_new is None else min(max(int(n_new[b]), 0), n)
            lo, hi = max(int(starts[b]), 0), min(int(starts[b]) + m, cap)
            for j in range(lo // BLOCK, (hi + BLOCK - 1) // BLOCK if hi > lo else 0):
                if (b, j) in dropped:
                    continue
                self.touched[b, j] = True
                r0, r1 = max(lo - j * BLOCK, 0), min(hi - j * BLOCK, BLOCK)
                first = j * BLOCK + r0 - int(starts[b])
                for held, scale, rows in ((self.k, self.ks, k), (self.v, self.vs, v)):
                    x = rows[b, first:first + r1 - r0].transpose(1, 0, 2)  # [Hkv, rows, D]
                    top = np.nanmax(np.where(np.isnan(x), 0, np.minimum(np.abs(x), BF16_MAX)), (1, 2))
                    sc = scale_of(top)
                    if r0:
                        sc = np.maximum(sc, scale[b, j])
                        old = E4M3[held[b, j, :, :r0]] * (scale[b, j] / sc)[:, None, None]
                        held[b, j, :, :r0] = e4m3(old)
                    held[b, j, :, r0:r1] = e4m3(x / sc[:, None, None])
                    held[b, j, :, r1:] = 0
                    scale[b, j] = sc
                s = E4M3[self.k[b, j, :, :r1]].sum(1) * self.ks[b, j][:, None]
                self.mean[b, j] = to_bf16((s / r1).astype(np.float32))

    def rows(self, which):
        """Dequantised rows [B, capacity, Hkv, 128]."""
        y, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        x = E4M3[y] * s[..., None, None]
        return x.transpose(0, 1, 3, 2, 4).reshape(self.B, -1, self.Hkv, D)


BF16_MAX = float(np.uint32(0x7f7f0000).view(np.float32))


def pools(model, table=None, n_pages=None, per=None, fill=0):
    """numpy pools (k, v uint8, k_scale, v_scale, k_mean fp64) of a model, dense (page =
    sequence) or by a block table [B, max_pages] of pages of `per` blocks; pages no table
    names hold `fill` bytes and NaN scales when fill is not 0."""
    B, nb, Hkv = model.B, model.nb, model.Hkv
    if table is None:
        table, n_pages, per = np.arange(B)[:, None], B, nb
    k = np.full((n_pages, Hkv, per, BLOCK * D), fill, dtype=np.uint8)
    v = k.copy()
    ks = np.full((n_pages, Hkv, per), math.nan if fill else 0.0)
    vs, mean = ks.copy(), np.full((n_pages, Hkv, per, D), math.nan if fill else 0.0)
    for b in range(B):
        for j in range(nb):
            pg, i = int(table[b, j // per]), j % per
            if not 0 <= pg < n_pages:
                continue
            k[pg, :, i], v[pg, :, i] = pack_k(model.k[b, j]), pack_v(model.v[b, j])
            ks[pg, :, i], vs[pg, :, i] = model.ks[b, j], model.vs[b, j]
            mean[pg, :, i] = model.mean[b, j]
    return (k.reshape(n_pages, Hkv, per * BLOCK, D), v.reshape(n_pages, Hkv, per * BLOCK, D), ks, vs,
            mean)


def rope(x, pos, theta=1e6):
    """x [..., n, 128] rotated to positions pos [n] (rotate-half)."""
    a = np.asarray(pos, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(64) / D)
    c, s = np.cos(a), np.sin(a)
    lo, hi = x[..., :64], x[..., 64:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def attend(q, k, v, pos, kv_len, w_pre, w0, bifocal=True, theta=1e6):
    """One query head q [128] at kv_len - 1 over keys k, v [n, 128] at positions pos [n].
    Returns (o, bound): the bound on |error| of each channel that the kernel's roundings
    allow.  A score's error is at most 4.5 half-steps of fp16 (the query's rotation, rounded
    once; the key's: cos/sin, product, sum; the fp32 sums are far below the half left) of
    sum (|q_i| + |q_i+64|)(|k_i| + |k_i+64|) / sqrt(d), which moves every weight by a factor
    of at most exp(2 delta); weights are rounded to fp16 once, the output to bf16 once."""
    o = np.zeros(D)
    keep = (pos < kv_len) & (pos >= 0)
    k, v, pos = k[keep], v[keep], pos[keep]
    if not len(pos):
        return o, np.zeros(D)
    G = max(1, -(-kv_len // w_pre)) if bifocal else 1
    qp = kv_len - 1
    near = (rope(k, pos, theta) @ rope(q[None], [qp], theta)[0]) / math.sqrt(D)
    far = (rope(k, pos // G, theta) @ rope(q[None], [qp // G], theta)[0]) / math.sqrt(D)
    s = np.where(qp - pos > w0, far, near) if bifocal else near
    p = np.exp(s - s.max())
    p /= p.sum()
    o = p @ v
    mag = (np.abs(k[:, :64]) + np.abs(k[:, 64:])) @ (np.abs(q[:64]) + np.abs(q[64:])) / math.sqrt(D)
    delta = 4.5 * U16 * mag.max()
    bound = (p @ np.abs(v - o)) * np.expm1(2 * delta) + U16 * (p @ np.abs(v)) + UBF * np.abs(o)
    return o, 1.01 * bound + 2.0 ** -40 * np.abs(v).sum(0) + 1e-37


def decode(q, model, lens, w_pre, w0, bifocal=True, blocks=None, theta=1e6):
    """q [B, Hq, 128] -> (o, bound), each [B, Hq, 128]; blocks [B, Hkv, n] lists or None."""
    B, Hq, _ = q.shape
    g = Hq // model.Hkv
    k, v = model.rows("k"), model.rows("v")
    o, bound = np.zeros((B, Hq, D)), np.zeros((B, Hq, D))
    cap = model.nb * BLOCK
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        for h in range(model.Hkv):
            pos = np.arange(n)
            if blocks is not None:
                js = [int(j) for j in blocks[b, h] if 0 <= j < model.nb]
                pos = np.concatenate([np.arange(j * BLOCK, (j + 1) * BLOCK) for j in js] or
                                     [np.zeros(0, dtype=np.int64)])
                pos = pos[pos < n].astype(np.int64)
            for i in range(g):
                o[b, h * g + i], bound[b, h * g + i] = attend(
                    q[b, h * g + i], k[b, pos, h], v[b, pos, h], pos, n, w_pre, w0, bifocal, theta)
    return o, bound


def select(scores, lens, n_select, w_local, n_first):
    B, Hkv, nb = scores.shape
    out = np.full((B, Hkv, n_select), -1, dtype=np.int32)
    for b in range(B):
        n = max(int(lens[b]), 0)
        last = min(nb, -(-n // BLOCK))
        for h in range(Hkv):
            def key(j):
                s = float(scores[b, h, j])
                always = j < n_first or j * BLOCK + BLOCK - 1 >= n - 1 - w_local
                return (0 if always else 1 if math.isnan(s) else 2, 0.0 if always or math.isnan(s)
                        else -s, j)
            chosen = sorted(sorted(range(last), key=key)[:n_select])
            out[b, h, :len(chosen)] = chosen
    return out
