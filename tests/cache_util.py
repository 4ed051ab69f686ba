"""Helpers of the compressed-cache tests: inputs, oracle values and tolerances derived from rounding."""
import numpy as np
import torch

from oracle import cache_oracle as C
from oracle import graphattn_oracle as O
from paper_2606_18954_amd import graphattn as G

BF16_HALF_STEP = 2.0 ** -8
FP16_HALF_STEP = 2.0 ** -11


def bits_of(t):
    """float64 values of a bf16 or float32 tensor."""
    return t.double().cpu().numpy()


def random_pool(rng, num_pages, Hkv, D, lo=-3, hi=3):
    """An MXFP4 pool of random codes, scales 2^lo .. 2^hi."""
    pool = rng.integers(0, 256, (num_pages, Hkv, 17 * D)).astype(np.uint8)
    pool[:, :, 16 * D:] = rng.integers(127 + lo, 128 + hi, (num_pages, Hkv, D))
    return pool


def poison_unused(pool, graph):
    """NaN scales (byte 255) in every slot that holds no token of a segment, and random codes."""
    D = pool.shape[2] // 17
    used = np.zeros(16 * pool.shape[0], dtype=bool)
    for s in range(graph.num_segments):
        for t in range(int(graph.seg_len[s])):
            page = int(graph.seg_pages[graph.seg_page_offsets[s] + t // 16])
            used[16 * page + t % 16] = True
    out = pool.copy()
    for w in np.nonzero(~used)[0]:
        for value in (False, True):
            for c in range(0, D, 32):
                out[w // 16, :, C.scale_place(int(w) % 16, c, D, value)] = 255
    return out


def draw_q(rng, rows, Hq, D, dtype="bf16"):
    q = torch.from_numpy(rng.standard_normal((rows, Hq, D)).astype(np.float32))
    return q.to(torch.bfloat16) if dtype == "bf16" else q


def output_bound(out, spread, vmax, out_f32=False):
    """How far a row's outputs may be off: every probability is rounded to bf16 (half a step of each
    weight: that share of the weighted |V|), every partial row to fp16 of the row's largest value, the
    result to bf16 unless float32 is asked for; sums in float32 over a few thousand terms."""
    b = BF16_HALF_STEP * spread + FP16_HALF_STEP * vmax + 2.0 ** -18 * vmax
    return b if out_f32 else b + BF16_HALF_STEP * (np.abs(out) + b)


def lse_bound(reach, D, lse):
    """Scores are float32 sums of D exact products of at most `reach` in total (half a step an
    addition, in the order of magnitude of the partial sums), converted to the log2 domain; the sum
    and its logarithm add a few steps of the result."""
    return (D + 8) * 2.0 ** -24 * reach + 2.0 ** -20 * (1.0 + np.abs(lse))


def check_attention(tag, out, lse, q, values, graph, Hq, Hkv, counts=None, rows=None, scale=None,
                    out_f32=False):
    oo, ol, spread, reach = C.attention(bits_of(q), values, graph, Hq, Hkv, counts, scale, rows)
    go, gl = bits_of(out), bits_of(lse)
    if rows is not None:
        go, gl = go[rows], gl[rows]
    assert np.isfinite(go).all() and np.isfinite(gl).all(), tag
    vmax = float(np.nanmax(np.abs(values)))
    off = np.abs(go - oo) / output_bound(oo, spread, vmax, out_f32)
    offl = np.abs(gl - ol) / lse_bound(reach, values.shape[-1], ol)
    print(f"[parity] {tag}: out {off.max():.3f} of its bound, lse {offl.max():.3f}", flush=True)
    assert off.max() <= 1.0, (tag, float(off.max()))
    assert offl.max() <= 1.0, (tag, float(offl.max()))


def mass_bound(q, values, graph, lse, Hq, Hkv, ref, decay, mass_in, counts=None):
    """float32 throughout: a score's error enters its weight as a factor (lse_bound's first term, and
    a few steps of score and lse in the log2 domain), sums of at most a few thousand positive terms."""
    reach = C.attention(bits_of(q), values, graph, Hq, Hkv, counts)[3]
    D = values.shape[-1]
    rel = (D + 8) * 2.0 ** -24 * reach + 2.0 ** -22 * (1.0 + reach + np.abs(lse[np.isfinite(lse)]).max())
    return (rel + 2.0 ** -16) * np.abs(ref) + 2.0 ** -22 * np.abs(decay * mass_in)
