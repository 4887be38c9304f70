"""Float64 reference of training device levels by reward (test infrastructure only).

The policy over a device's levels: pixel r draws level j with probability
softmax(logits_r)_j; logits [R, K], actions [S, R], a negative action standing
for no choice.  The optimiser: the 2-norm over several gradients and AdamW,
whose moments are formed in float32, each product and sum rounded, and stored
as they are or in 8 bits.
"""

from __future__ import annotations

import numpy as np

BLOCK = 256


def log_softmax(logits: np.ndarray) -> np.ndarray:
    x = logits.astype(np.float64)
    with np.errstate(invalid="ignore"):
        d = x - x.max(axis=-1, keepdims=True)
        return d - np.log(np.exp(d).sum(axis=-1, keepdims=True))


def policy_draw(logits: np.ndarray, noise: np.ndarray) -> np.ndarray:
    """First level of the largest float32 score; scores that are NaN left out, 0 where all are."""
    score = logits.astype(np.float32) + noise.astype(np.float32)
    score = np.where(np.isnan(score), -np.inf, score)
    return score.argmax(axis=-1).astype(np.int32)


def policy_logp(logits: np.ndarray, actions: np.ndarray) -> np.ndarray:
    k = logits.shape[-1]
    lp = np.take_along_axis(log_softmax(logits), np.clip(actions, 0, k - 1).T, axis=1).T
    return np.where(actions < 0, 0.0, np.where(actions >= k, np.nan, lp))


def policy_loss(logits, actions, old_logp, advantages, ref_logp=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                entropy_coef=0.0, scale=1.0):
    """(loss, terms [4], dL/dlogits, size of the gradient's parts): the last is what the terms of a
    gradient's value add up to without their signs, by which a rounding error is judged."""
    f = lambda v: float(np.float32(v))  # noqa: E731
    lo, hi, kl_c, ent_c, scale = 1.0 - f(clip_low), 1.0 + f(clip_high), f(kl_coef), f(entropy_coef), f(scale)
    s, r = actions.shape
    adv = np.asarray(advantages, np.float64)
    adv = np.broadcast_to(adv if adv.ndim == 2 else adv[:, None], (s, r))
    logp = log_softmax(logits)
    p = np.exp(logp)
    plogp = np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0)
    entropy = -plogp.sum(-1)
    grad = np.zeros(logits.shape)
    size = np.zeros(logits.shape)
    terms = np.zeros(4)
    sizes = np.zeros(4)
    for row in range(r):
        total, rough, made = 0.0, 0.0, 0
        for i in range(s):
            a = int(actions[i, row])
            if a < 0:
                continue
            made += 1
            lp = logp[row, a]
            ratio = np.exp(lp - float(old_logp[i, row]))
            value = min(ratio * adv[i, row], min(max(ratio, lo), hi) * adv[i, row])
            over = ratio > hi if adv[i, row] >= 0 else ratio < lo
            g = 0.0 if over else -ratio * adv[i, row]
            q = 0.0
            if ref_logp is not None:
                d = float(ref_logp[i, row]) - lp
                q = np.expm1(d) - d
                g -= kl_c * np.expm1(d)
            here = np.array([-value, q, entropy[row], float(over)])
            terms += here
            sizes += np.abs(here) + np.array([abs(adv[i, row]) * ratio, 0, 0, 0])
            total += g
            bound = ratio * abs(adv[i, row]) + (kl_c * (1 + np.exp(d)) if ref_logp is not None else 0.0)
            rough += bound
            grad[row, a] += g
            size[row, a] += bound
        if made:
            grad[row] -= p[row] * total
            size[row] += p[row] * rough
            extra = ent_c * made * (plogp[row] + p[row] * entropy[row])
            grad[row] += extra
            size[row] += ent_c * made * (np.abs(plogp[row]) + p[row] * (entropy[row] + 1))
    loss = terms[0] + kl_c * terms[1] - ent_c * terms[2]
    return loss * scale, terms * scale, grad * scale, size * scale, sizes * scale


def grad_norm(grads) -> float:
    return float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))


def mix(x: np.ndarray) -> np.ndarray:
    """The 32-bit hash of the random bits."""
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed: int, tensor: int, index: np.ndarray) -> np.ndarray:
    index = np.asarray(index, np.uint64)
    key = mix(mix(np.uint64((seed + 0x9E3779B9 * tensor) & 0xFFFFFFFF)) + (index >> np.uint64(32)))
    return mix((index & np.uint64(0xFFFFFFFF)) + key)


def code_values(least: int, count: int) -> np.ndarray:
    """What the codes 0 .. count - 1 stand for, over twice the scale."""
    c = np.arange(count)
    e, f = c >> 3, c & 7
    return np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 1 + least), f / 8 * 2.0 ** least)


def decode(codes_m, codes_v, scales):
    """float64 moments of 8-bit codes; scales [blocks, 2]."""
    n = codes_m.size
    u = np.repeat(scales.astype(np.float64), BLOCK, axis=0)[:n]
    m = code_values(-14, 128)[codes_m & 127] * 2 * u[:, 0]
    return np.where(codes_m & 128, -m, m), code_values(-30, 256)[codes_v] * 2 * u[:, 1]


def _encode(x, bits, least):
    """(codes of the magnitudes of float32 values, scales): the code below the value, or the next one where the
    place between the two and 20 random bits reach one."""
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK, np.float32)
    pad[:n] = np.abs(x)
    top = pad.reshape(-1, BLOCK).max(axis=1)
    e = np.maximum(top.view(np.int32) >> 23, 27)
    scale = np.where(e < 253, np.ldexp(1.0, e - 127), np.nan).astype(np.float32)
    codes = np.zeros(pad.size, np.int64)
    values = code_values(least, 257)
    ok = np.repeat(e < 253, BLOCK)
    y = np.zeros(pad.size)
    y[ok] = pad[ok].astype(np.float64) / np.repeat(np.ldexp(1.0, e - 126), BLOCK)[ok]
    small = y < 2.0 ** least
    y = np.where(small, (y + 2.0 ** least).astype(np.float32).astype(np.float64) - 2.0 ** least, y)
    low = np.searchsorted(values, y, side="right") - 1
    place = (y - values[low]) / (values[low + 1] - values[low])
    r = np.zeros(pad.size)
    r[:n] = bits.astype(np.float64) / 2 ** 20
    codes = np.where(ok, low + (place + r >= 1.0), 0)
    return codes[:n], scale


def encode(m, v, bits):
    """(codes of m, codes of v, scales) of float32 moments with 32 random bits each."""
    cm, sm = _encode(m, bits & np.uint64(0xFFFFF), -14)
    cv, sv = _encode(v, bits >> np.uint64(12), -30)
    cm = np.where((m < 0) & np.repeat(np.isfinite(sm), BLOCK)[:m.size], cm | 128, cm)
    cv = np.where((v > 0) & (cv == 0) & np.repeat(np.isfinite(sv), BLOCK)[:v.size], 1, cv)
    return cm.astype(np.uint8), cv.astype(np.uint8), np.stack([sm, sv], 1)


def adamw(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, norm=None, max_norm=np.inf):
    """(p in float64, m and v in float32) after one step on float32 arrays; norm: of all gradients."""
    f = np.float32
    b1, b2 = f(beta1), f(beta2)
    c1, c2 = f(1.0 - float(b1)), f(1.0 - float(b2))
    g = g.astype(f)
    if norm is not None:
        if not np.isfinite(norm):
            return p.astype(np.float64), m, v
        g = g * (f(max_norm) / f(norm) if f(norm) > f(max_norm) else f(1.0))
    m = m * b1 + g * c1
    v = v * b2 + (g * g) * c2
    lr, wd = float(f(lr)), float(f(weight_decay))
    up = (m.astype(np.float64) / (1.0 - float(b1) ** step)
          / (np.sqrt(v.astype(np.float64) / (1.0 - float(b2) ** step)) + float(f(eps))))
    return p.astype(np.float64) * (1.0 - lr * wd) - lr * up, m, v
