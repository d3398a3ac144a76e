"""Inputs of the cache and attention tests: pools of arbitrary codes, tables of pages, lengths."""
import numpy as np

BLOCK = {"nvfp4": 16, "mxfp4": 32}


def pool(rng, fmt, pages, H, page, D):
    """Arbitrary codes under scales of a realistic range: codes, scales, S."""
    codes = rng.integers(0, 256, (pages, H, page, D // 2)).astype(np.uint8)
    if fmt == "nvfp4":
        return codes, rng.integers(0x20, 0x70, (pages, H, page, D // 16)).astype(np.uint8), (rng.random(H) * 0.01 + 0.003).astype(np.float32)
    return codes, rng.integers(122, 128, (pages, H, page, D // 32)).astype(np.uint8), None


def table(rng, B, cols, pages):
    """Distinct pages in any order."""
    return rng.permutation(pages)[:B * cols].reshape(B, cols).astype(np.int32)


def offsets_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
