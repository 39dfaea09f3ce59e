"""Inputs and plain 64-bit definitions for the tests of the calls that take
several tokens a sequence: paged requests, and rotary positions by complex
numbers."""

import numpy as np
import torch

BS = 16


def cfg_of(hq, hkv, d, qk_norm=0, layers=1, hidden=64, ffn=64):
    return dict(num_layers=layers, hidden=hidden, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, ffn_dim=ffn, qkv_bias=0,
                qk_norm=qk_norm, rms_eps=1e-6, qk_norm_eps=1e-6, rope_theta=1e4, block_size=BS)


class Handle:
    """A handle for single calls: no pool, caches of one or more regions filled with `fill`."""

    def __init__(self, lib, cfg, max_seq_len, nblk=0, regions=1, fill=0.0):
        self.lib, self.cfg, self.nblk = lib, cfg, nblk
        self.h = lib.sidp_create(lib.make_config(cfg, 1, max_seq_len))
        hkv, d = cfg["num_kv_heads"], cfg["head_dim"]
        if nblk:
            self.k = torch.full((regions, nblk, hkv, d // 8, BS, 8), fill, dtype=torch.bfloat16, device="cuda")
            self.v = torch.full((regions, nblk, hkv, d, BS), fill, dtype=torch.bfloat16, device="cuda")
            lib.sidp_kv_attach(self.h, self.k, self.v, nblk, regions)

    def sync(self):
        self.lib.sidp_sync(self.h)

    def close(self):
        self.lib.sidp_destroy(self.h)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # caches as [slot][head][d]
    def keys(self, region=0):
        return self.k[region].permute(0, 3, 1, 2, 4).reshape(self.nblk * BS, self.cfg["num_kv_heads"], -1)

    def values(self, region=0):
        return self.v[region].permute(0, 3, 1, 2).reshape(self.nblk * BS, self.cfg["num_kv_heads"], -1)


def turn(x, pos, freqs, scale, interleaved):
    """x [rows, heads, D] in float64: each pair as a complex number times scale e^(i pos w)."""
    x = np.array(x, dtype=np.float64)
    n = len(freqs)
    z = np.exp(1j * np.asarray(pos, np.float64)[:, None] * np.asarray(freqs)[None, :])[:, None, :] * scale
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    w = (a + 1j * b) * z
    if interleaved:
        x[..., 0:2 * n:2], x[..., 1:2 * n:2] = w.real, w.imag
    else:
        x[..., :n], x[..., n:2 * n] = w.real, w.imag
    return x


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")
