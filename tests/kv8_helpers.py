"""The 8-bit cache in plain numpy: codes and scales by their definition, and a
handle with such a cache attached."""

import numpy as np
import torch

from rows_helpers import BS, Handle

E4M3_MAX = 448.0


def e4m3_values():
    """The value of each of the 256 codes: sign, 4 bits of exponent (bias 7), 3 bits behind the point; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7.0), m / 8 * 2.0 ** -6)
    v = np.where(c & 127 == 127, np.nan, v)
    return np.where(c & 128, -v, v)


E4M3 = e4m3_values()


def to_e4m3(x):
    """Nearest codes of |x| <= 448, ties to the even code."""
    mags = E4M3[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(mags, a), 1, 126)
    lo = hi - 1
    dl, dh = a - mags[lo], mags[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def scale_of(x, kind):
    """fp32 scales of vectors along the last axis."""
    x = np.asarray(x, np.float64)
    most = np.max(np.abs(x), -1)
    with np.errstate(divide="ignore", invalid="ignore"):
        if kind == "e4m3":
            m, e = np.frexp(most)  # 448 = 0.875 * 2^9
            s = np.where(most > 0, np.ldexp(1.0, np.maximum(e - 9 + (m > 0.875), -126)), 2.0 ** -126)
        else:
            s = np.maximum((most.astype(np.float32) / np.float32(127)).astype(np.float64), 2.0 ** -126)
    return np.where(np.isfinite(x).all(-1), s, np.nan)


def codes_of(x, scale, kind):
    x, scale = np.asarray(x, np.float64), np.asarray(scale, np.float64)[..., None]
    ok = np.isfinite(scale)
    z = np.where(ok, np.where(ok, x, 0) / np.where(ok, scale, 1), 0)
    if kind == "e4m3":
        return np.where(ok, to_e4m3(z), 0).astype(np.uint8)
    # the quotient is rounded to fp32 first, as the definition divides fp32 by fp32
    return np.rint(z.astype(np.float32)).astype(np.int8).view(np.uint8)


def values_of(codes, kind):
    return E4M3[codes] if kind == "e4m3" else codes.view(np.int8).astype(np.float64)


def half_step(x, scale, kind):
    """The largest distance of a value from its code's: half a step."""
    scale = np.asarray(scale, np.float64)[..., None]
    if kind == "int8":
        return np.broadcast_to(scale / 2, np.shape(x))
    z = np.abs(x) / scale
    return 2.0 ** (np.floor(np.log2(np.maximum(z, 2.0 ** -6))) - 4) * scale


class Handle8(Handle):
    """A handle with an 8-bit cache of `regions` regions, every byte of it `fill` (codes) and `scale` at the start."""

    def __init__(self, lib, cfg, max_seq_len, nblk, kind, regions=1, fill=0x7f, scale=float("nan"), bf16_blocks=0):
        super().__init__(lib, cfg, max_seq_len, bf16_blocks, regions)
        self.kind, self.nblk8 = kind, nblk
        hkv, d = cfg["num_kv_heads"], cfg["head_dim"]
        self.k8 = torch.full((regions, nblk, hkv, d // 16, BS, 16), fill, dtype=torch.uint8, device="cuda")
        self.v8 = torch.full((regions, nblk, hkv, d, BS), fill, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((regions, nblk, hkv, 2, BS), scale, device="cuda")
        lib.sidp_kv8_attach(self.h, {"e4m3": lib.SIDP_KV_E4M3, "int8": lib.SIDP_KV_INT8}[kind], self.k8, self.v8, self.scales,
                            nblk, regions)

    # as [slot][head][d], and scales as [slot][head]
    def key_codes(self, region=0):
        return self.k8[region].permute(0, 3, 1, 2, 4).reshape(self.nblk8 * BS, self.cfg["num_kv_heads"], -1).cpu().numpy()

    def value_codes(self, region=0):
        return self.v8[region].permute(0, 3, 1, 2).reshape(self.nblk8 * BS, self.cfg["num_kv_heads"], -1).cpu().numpy()

    def key_scales(self, region=0):
        return self.scales[region][:, :, 0].permute(0, 2, 1).reshape(self.nblk8 * BS, -1).double().cpu().numpy()

    def value_scales(self, region=0):
        return self.scales[region][:, :, 1].permute(0, 2, 1).reshape(self.nblk8 * BS, -1).double().cpu().numpy()

    def put(self, region, slots, k, v):
        """Keys and values [rows, head, d] (numpy, 64 bits) coded by the definition into the given slots; returns what they are held as."""
        held = []
        slots = torch.as_tensor(np.asarray(slots), dtype=torch.long, device="cuda")
        blk, off = slots // BS, slots % BS
        for which, x in ((0, k), (1, v)):
            s = scale_of(x, self.kind)
            c = codes_of(x, s, self.kind)
            held.append(values_of(c, self.kind) * s[..., None])
            c, s32 = torch.as_tensor(c).cuda(), torch.as_tensor(s.astype(np.float32)).cuda()
            if which == 0:
                self.k8[region][blk, :, :, off, :] = c.view(len(x), x.shape[1], -1, 16)
            else:
                self.v8[region][blk, :, :, off] = c
            self.scales[region][blk, :, which, off] = s32
        return held
