"""CPU oracle of the operators over the tokens of long videos: plain definitions in numpy float64, one loop per thing that the
definition loops over. Nothing here is shared with the product."""
import math

import numpy as np


# ---- rotary positions ------------------------------------------------------------------------------------------------
def rope_pairs(axes, layout):
    """(first channel, second channel, axis, index of the pair within its axis) of every pair."""
    out, at = [], 0
    for a, D in enumerate(axes):
        for i in range(D // 2):
            out.append((at + i, at + D // 2 + i, a, i) if layout == "half" else (at + 2 * i, at + 2 * i + 1, a, i))
        at += D
    return out


def rope_frequency(D, i, base=10000.0, scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0):
    """Radians a position of pair i of an axis of D channels."""
    if scaling == "base" and D > 2:
        base = base * factor ** (D / (D - 2))
    w = base ** (-2.0 * i / D)
    if scaling == "linear":
        w /= factor
    if scaling == "parts":
        turns = orig_len * w / (2.0 * math.pi)
        keep = min(max((turns - beta_slow) / (beta_fast - beta_slow), 0.0), 1.0)
        w *= keep + (1.0 - keep) / factor
    return w


def rope(x, pos, axes, layout="half", inverse=False, **scaling):
    """x [B, T, H, d], pos integers [B, T, axes]."""
    y = np.array(x, dtype=np.float64)
    amp = 0.1 * math.log(scaling["factor"]) + 1.0 if scaling.get("scaling") == "parts" and scaling["factor"] > 1 else 1.0
    for u, v, a, i in rope_pairs(axes, layout):
        angle = np.asarray(pos)[:, :, a].astype(np.float64) * rope_frequency(axes[a], i, **scaling)
        c, s = (amp * np.cos(angle))[:, :, None], (amp * np.sin(angle))[:, :, None]
        if inverse:
            s = -s
        y[..., u], y[..., v] = x[..., u] * c - x[..., v] * s, x[..., u] * s + x[..., v] * c
    return y


# ---- attention over selected blocks ----------------------------------------------------------------------------------
def _lens(lens, B, T):
    return [T] * B if lens is None else [min(max(int(n), 0), T) for n in lens]


def block_means(k, block, k_len=None):
    """k [B, Tk, Hkv, d] -> [B, Hkv, d, blocks]"""
    B, Tk, Hkv, d = k.shape
    out = np.zeros((B, Hkv, d, -(-Tk // block)))
    for b, n in enumerate(_lens(k_len, B, Tk)):
        for j in range(-(-n // block)):
            out[b, :, :, j] = k[b, j * block:min(n, (j + 1) * block)].astype(np.float64).mean(axis=0)
    return out


def block_select(q, means, Tk, keep, block, q_block, sink=0, window=-1, q_pos0=0, q_len=None, k_len=None):
    B, Tq, H, d = q.shape
    Hkv, nq = means.shape[1], -(-Tq // q_block)
    out = np.full((B, H, nq, keep), -1, dtype=np.int32)
    for b, (ql, kl) in enumerate(zip(_lens(q_len, B, Tq), _lens(k_len, B, Tk))):
        for h in range(H):
            for g in range(-(-ql // q_block)):
                mean = q[b, g * q_block:min(ql, (g + 1) * q_block), h].astype(np.float64).mean(axis=0)
                p0 = q_pos0 + g * q_block
                p1 = q_pos0 + min(ql, (g + 1) * q_block) - 1
                ranked = []
                for j in range(-(-kl // block)):
                    s = float(mean @ means[b, h * Hkv // H, :, j])
                    forced = j < sink or (window >= 0 and p0 // block - window <= j <= p1 // block + window)
                    ranked.append((0 if forced else 2 if math.isnan(s) else 1, 0.0 if forced or math.isnan(s) else -s, j))
                best = sorted(j for _, _, j in sorted(ranked)[:keep])
                out[b, h, g, :len(best)] = best
    return out


def listed_blocks(entries, block, keys):
    """A list ends at its first entry that is no block with a key or does not ascend."""
    out = []
    for e in entries:
        if e < 0 or e * block >= keys or (out and e <= out[-1]):
            break
        out.append(int(e))
    return out


def block_attention(q, k, v, index, block, q_block, q_len=None, k_len=None, scale=None):
    """out [B, Tq, H, d], and the two sums that error bounds are made of: sum w |v| and the largest sum |q k| of a query."""
    B, Tq, H, d = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, weight, dot = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, Tq, H, 1))
    for b, (ql, kl) in enumerate(zip(_lens(q_len, B, Tq), _lens(k_len, B, Tk))):
        for h in range(H):
            kb, vb = k[b, :, h * Hkv // H].astype(np.float64), v[b, :, h * Hkv // H].astype(np.float64)
            for g in range(-(-ql // q_block)):
                r = slice(g * q_block, min(ql, (g + 1) * q_block))
                keys = [t for j in listed_blocks(index[b, h, g], block, kl) for t in range(j * block, min(kl, (j + 1) * block))]
                if not keys:
                    continue
                qr = q[b, r, h].astype(np.float64)
                s = scale * (qr @ kb[keys].T)
                w = np.exp(s - s.max(axis=1, keepdims=True))
                w /= w.sum(axis=1, keepdims=True)
                out[b, r, h], weight[b, r, h] = w @ vb[keys], w @ np.abs(vb[keys])
                dot[b, r, h, 0] = scale * (np.abs(qr) @ np.abs(kb[keys]).T).max(axis=1)
    return out, weight, dot


# ---- quantised cache entries -----------------------------------------------------------------------------------------
def magnitudes(fmt):
    """Every magnitude that a code stands for, by ascending code."""
    if fmt == "mxint8":
        return np.arange(128.0)
    if fmt == "mxfp4":
        return np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    small = [f / 8 * 2.0 ** -6 for f in range(8)]
    return np.array(small + [(1 + f / 8) * 2.0 ** (e - 7) for e in range(1, 16) for f in range(8)][:-1])


FLOAT_MAX = (2.0 - 2.0 ** -23) * 2.0 ** 127


def entry(x, fmt):
    """x [rows, cols] float32 -> (values the entry stands for, scale exponents [rows, groups]; exponent 128 marks no number). A code is
    the nearest one whose value a float holds."""
    rows, cols = x.shape
    steps = magnitudes(fmt)
    top = steps[-1]
    values, exps = np.zeros((rows, cols)), np.zeros((rows, -(-cols // 32)), dtype=np.int64)
    for r in range(rows):
        for g in range(exps.shape[1]):
            v = np.asarray(x[r, g * 32:(g + 1) * 32], dtype=np.float64)
            if not np.all(np.isfinite(v)):
                values[r, g * 32:(g + 1) * 32], exps[r, g] = np.nan, 128
                continue
            e = -127
            while np.abs(v).max(initial=0.0) > top * 2.0 ** e:
                e += 1
            exps[r, g] = e
            held = steps[steps * 2.0 ** e <= FLOAT_MAX]
            for i, a in enumerate(np.abs(v) / 2.0 ** e):
                up = int(np.searchsorted(held, a))
                if up == 0 or up == len(held):
                    code = min(up, len(held) - 1)
                else:
                    hi, lo = steps[up] - a, a - steps[up - 1]
                    code = up if hi < lo or (hi == lo and up % 2 == 0) else up - 1
                values[r, g * 32 + i] = math.copysign(steps[code], v[i]) * 2.0 ** e
    return values, exps
