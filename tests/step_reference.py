"""Plain 64-bit references of rotary rows, the step between blocks and the rules
on logits.  Test infrastructure only."""

import math

import torch


def frequencies(rotary_dim, base=10000.0, scaling=None, factor=1.0, original=0, low=1.0, high=32.0):
    half, out = rotary_dim // 2, []
    if scaling == "base":
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    for i in range(half):
        theta = base ** (-2 * i / rotary_dim)
        share = 1.0
        if scaling == "linear":
            share = 0.0
        elif scaling == "rotations":
            share = (original * theta / (2 * math.pi) - low) / (high - low)
        elif scaling == "dims":
            def pair(turns):
                return rotary_dim * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), half - 1)
            share = 1 - (i - first) / max(last - first, 0.5)
        share = min(max(share, 0.0), 1.0)
        out.append(share * theta + (1 - share) * theta / factor)
    return out


def rotate(x, positions, theta, interleaved, axes=None, amplitude=1.0, weight=None, eps=1e-6,
           offset=0.0, transposed=False):
    """(y, size) of rows x [..., heads, d] in 64 bits; size [..., heads, d] is what
    an error of one part is relative to: |x| + |its pair| as they are turned."""
    x = x.double()
    D, d = 2 * len(theta), x.shape[-1]
    if weight is not None:
        x = x / ((x * x).sum(-1, keepdim=True) / d + eps).sqrt() * (offset + weight.double())
    p = positions.double()
    p = p[..., None].expand(*p.shape, D // 2) if axes is None else torch.stack([p[a] for a in axes], -1)
    angle = (p * torch.tensor(theta, dtype=torch.float64, device=x.device)).unsqueeze(-2)
    if transposed:
        angle = -angle
    a, b = ((x[..., 0:D:2], x[..., 1:D:2]) if interleaved else (x[..., :D // 2], x[..., D // 2:D]))
    c, s = amplitude * angle.cos(), amplitude * angle.sin()
    ya, yb, size = a * c - b * s, a * s + b * c, abs(amplitude) * (a.abs() + b.abs())

    def place(u, v):
        t = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
        return torch.cat((t, x[..., D:]), -1)

    return place(ya, yb), place(size, size).abs()


def normed(v, kind, weight, bias, eps, offset):
    """The norm in 64 bits."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    y = v / ((v * v).mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        y = y * (offset + weight.double())
    return y if bias is None else y + bias.double()


GATES = {"linear": lambda g: g, "sigmoid": torch.sigmoid, "tanh": torch.tanh,
         "silu": lambda g: g * torch.sigmoid(g)}


def rules(x, history, prompt, repetition=1.0, frequency=0.0, presence=0.0, biases=None, allowed=None):
    """One row [V] on the CPU before the temperature, in fp32 with each step
    rounded as written; history: a list of tokens, the first `prompt` the prompt;
    biases: {token: value}; allowed [V] bool."""
    x, V = x.float().clone(), x.numel()
    one = torch.float32
    rep, freq, pres = (torch.tensor(t, dtype=one) for t in (repetition, frequency, presence))
    count = {}
    for i, t in enumerate(history):
        if 0 <= t < V:
            count[t] = count.get(t, 0) + (i >= prompt)
    for t, n in count.items():
        x[t] = x[t] / rep if x[t] > 0 else x[t] * rep
        if n:
            x[t] = x[t] - (freq * torch.tensor(float(n), dtype=one) + pres)
    for t, b in (biases or {}).items():
        x[t] = x[t] + torch.tensor(b, dtype=one)
    if allowed is not None:
        x[~allowed] = -math.inf
    return x


def best_of(x):
    """(token, or -1) of a row under the rules: the lowest of the largest."""
    y = torch.where(x.isnan(), torch.tensor(-math.inf), x)
    top = y.max()
    return -1 if top == -math.inf else int((y == top).nonzero()[0])
