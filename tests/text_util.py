"""Helpers of the language-model operators' tests: types, roundings, inputs on the device (no method arithmetic)."""
import numpy as np

TYPES = ("float32", "bfloat16", "float16")
# half a step of each type relative to the value, and half the distance of its smallest values
HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
HALF_LEAST = {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}


def stored(torch, x, dtype):
    """x rounded to the type: (the device tensor, the rounded values in fp64)."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(getattr(torch, dtype))
    return t.cuda(), t.double().numpy()


def rows_in(torch, rows, width, pitch, dtype, offset=0, fill=float("nan")):
    """A (rows, width) view at `pitch`, `offset` elements into an allocation filled with `fill`, and the whole allocation."""
    flat = torch.full((rows * pitch + offset,), fill, dtype=getattr(torch, dtype), device="cuda")
    return flat[offset:].view(rows, pitch)[:, :width], flat


def tokens_of(rng, n, T, V, pad=0.2):
    """Frequent and rare tokens, some padding on both sides of the vocabulary."""
    t = np.floor(np.exp(rng.uniform(0, np.log(V + 1), (n, T)))).astype(np.int64) - 1
    t = np.clip(t, 0, V - 1)
    t[rng.uniform(size=(n, T)) < pad] = -1
    t[rng.uniform(size=(n, T)) < pad / 4] = V
    return t.astype(np.int32)
