"""The target's choices after penalties, biases and a grammar, token by token (test infrastructure).

Verification leaves the output distribution of the target model unchanged (paper, Section 2.3), whatever that model's
sampling settings are: penalties for tokens that have occurred, additive biases, a mask of what a grammar allows.  Each
slot of a draft tree is a text of its own, so the tokens on its path count as well."""
from __future__ import annotations

import numpy as np

f32 = np.float32


def process_row(logits: np.ndarray, context, prompt_len: int, path, repetition, presence, frequency, bias, allowed) -> np.ndarray:
    """logits float32 [V]; context, path: token ids; bias: list of (token, value); allowed: bool [V] or None."""
    V = len(logits)
    every = [t for t in list(context) + list(path) if 0 <= t < V]
    made = np.zeros(V, dtype=np.int64)
    for i, t in enumerate(context):
        if i >= prompt_len and 0 <= t < V:
            made[t] += 1
    for t in path:
        if 0 <= t < V:
            made[t] += 1
    x = logits.astype(f32).copy()
    with np.errstate(all="ignore"):
        for t in set(every):
            x[t] = x[t] / f32(repetition) if x[t] > 0 else x[t] * f32(repetition)
        for t in np.nonzero(made)[0]:
            x[t] = f32(x[t] - f32(f32(frequency) * f32(made[t])))
            x[t] = f32(x[t] - f32(presence))
        for t, v in dict(bias).items():                        # the last entry of a token counts
            if 0 <= t < V:
                x[t] = f32(x[t] + f32(v))
    if allowed is not None:
        x[~allowed] = -np.inf
    return x


def choose(x: np.ndarray) -> int:
    """The largest value's token, the lowest one of equals; -1 if nothing is above -inf."""
    y = np.where(np.isnan(x), -np.inf, x)
    return -1 if y.max() == -np.inf else int(np.argmax(y))
