"""Inputs shared by the tests of the 8-bit cache."""
import numpy as np
import torch

KV_DTYPE = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def trees(rng, B, N, full=False):
    """(num_nodes, parent): random trees, a request in four shorter than N slots."""
    parent = np.full((B, N), -1, np.int32)
    nn = np.zeros(B, np.int32)
    for i in range(B):
        nn[i] = N if full or rng.random() < 0.75 else int(rng.integers(1, N + 1))
        for j in range(1, nn[i]):
            parent[i, j] = int(rng.integers(max(0, j - 4), j))
    return nn, parent


def pages(rng, positions, page, spare=3):
    """(page_table, total): a shuffled private page for every page of every request, unused entries out of range."""
    need = [max(1, -(-int(p) // page)) for p in positions]
    total = sum(need) + spare
    perm = rng.permutation(total)
    pt = np.full((len(need), max(need)), 1 << 30, np.int32)
    at = 0
    for i, c in enumerate(need):
        pt[i, :c] = perm[at:at + c]
        at += c
    return pt, total


def cache(rng, kv, total, Hkv, page, block, spread=0.3, pow2=False):
    """(codes uint8 [total, Hkv, page, 128], scale float32): values around N(0, 1)."""
    most = 448.0 if kv == "e4m3" else 57344.0
    x = torch.from_numpy(rng.standard_normal((total, Hkv, page, 128)).astype(np.float32) * (most / 4))
    codes = x.clamp(-most, most).to(KV_DTYPE[kv]).view(torch.uint8).numpy().copy()
    scale = np.exp(spread * rng.standard_normal((total, Hkv, page // block))) * 4 / most
    if pow2:
        scale = 2.0 ** np.round(np.log2(scale))
    return codes, scale.astype(np.float32)


def to_device(codes, kv, token_major, dev="cuda:0"):
    """The pool as a [pages, Hkv, page, D] view, stored head by head or token by token."""
    t = torch.from_numpy(np.ascontiguousarray(codes)).to(dev)
    if token_major:
        t = t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    return t.view(KV_DTYPE[kv]) if kv != "bf16" else t


def codes_of(pool):
    return pool.view(torch.uint8).cpu().numpy()
