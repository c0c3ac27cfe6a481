"""Plain 64-bit statements of the operators under a rule: scaled rotary frequencies and tables, normed and rotated heads, attention
with a cap, a bias by distance, a window, documents and open keys."""
import math
from fractions import Fraction

import torch

FAR = (1 << 31) - 1

# 1 / 2 pi to 60 digits
PER_TURN = Fraction(159154943091895335768883763372514362034459645740456448747667, 10 ** 60)


def frequencies(dims, base, kind="", factor=1.0, original=0, low=1.0, high=32.0):
    out = []
    for i in range(dims // 2):
        b = base * factor ** (dims / (dims - 2)) if kind == "ntk" else base
        t = math.exp(-2.0 * i / dims * math.log(b))
        if kind == "linear":
            t /= factor
        if kind == "parts":
            g = min(1.0, max(0.0, (original * t / (2 * math.pi) - low) / (high - low)))
            t = (1 - g) * t / factor + g * t
        out.append(t)
    return out


def cos_sin(position, freq, amplitude=1.0):
    """Of the exact product, whole turns taken off before it becomes a float."""
    turns = Fraction(freq) * position * PER_TURN
    turns -= round(turns)
    quarter = round(4 * turns)
    x = float(turns - Fraction(quarter, 4)) * 2 * math.pi
    c, s = [(math.cos(x), math.sin(x)), (-math.sin(x), math.cos(x)), (-math.cos(x), -math.sin(x)), (math.sin(x), -math.cos(x))][quarter % 4]
    return c * amplitude, s * amplitude


def turned(x, positions, gain, eps, rope, interleaved):
    """Heads x [rows][heads][dh] in 64 bits, normed and rotated, and the magnitudes that scale the error of each value."""
    y = x.double()
    if gain is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double()
    mag = y.abs()
    if rope is not None:
        cos, sin = rope[0].double()[positions][:, None], rope[1].double()[positions][:, None]
        half = cos.shape[-1]
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        u, w = y[..., a], y[..., b]
        y, mag = y.clone(), mag.clone()
        y[..., a], y[..., b] = u * cos - w * sin, w * cos + u * sin
        mag[..., a], mag[..., b] = (u * cos).abs() + (w * sin).abs(), (w * cos).abs() + (u * sin).abs()
    return y, mag


def seen(p, n, lo=0, window=0, opened=0):
    """Which of a sequence's n keys the row of key p sees."""
    j = torch.arange(n)
    if p < 0:
        return torch.zeros(n, dtype=torch.bool)
    if window:
        lo = max(lo, p - window + 1)
    return (j < opened) | ((j >= lo) & (j <= p))


def attend(q, k, v, rows, cap=0.0, slopes=None, window=0):
    """q [n][heads][dh] over k, v [KV heads][len][dh]; rows: (p, first key, open keys) of each. Outputs in 64 bits and sum p |v|."""
    n, hq, dh = q.shape
    G, ln = hq // k.shape[0], k.shape[1]
    out, mag = torch.zeros(n, hq, dh, dtype=torch.float64), torch.zeros(n, hq, dh, dtype=torch.float64)
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    j = torch.arange(ln)
    for i, (p, lo, opened) in enumerate(rows):
        m = seen(p, ln, lo, window, opened)
        if not m.any():
            continue
        d = (p - j[m]).abs().double()
        for h in range(hq):
            s = k[h // G, m] @ q[i, h] / math.sqrt(dh)
            if cap:
                s = cap * torch.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[h]) * (d - d.min())
            w = torch.softmax(s, 0)
            out[i, h], mag[i, h] = w @ v[h // G, m], w @ v[h // G, m].abs()
    return out, mag


def check(got, want, mag, what):
    """fp32: a score of dh = 128 products of fp32 sums is off by some sqrt(128) 2^-24 sum |q k| / sqrt(dh), with queries of deviation 1.5
    about 8e-6; a cap's tanh by 2^-22 of a score of at most 10, 2.4e-6; a distance times its slope, of at most 25 where the key
    counts, by 2^-24 of it twice, 3e-6. A probability moves by as much of itself: 3e-5 of sum p |v| holds the three twice. bf16: at most
    half a step, 2^-8, of each rounded probability and 2^-8 of the output, beside that."""
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    bound = 3e-5 * mag + 1e-30
    if what[0] == "bf16":
        bound = bound + 2 ** -8 * (want.abs() + 1.01 * mag)
    worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (what, worst)
