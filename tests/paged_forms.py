"""Decoding steps from pages that between them reach every form of the kernels, and how closely a step has to meet float64.

A step of bf16 rows takes every vector into its products as a bf16 head and a bf16 remainder, which leaves 2^-16 of an element at most
and 2^-18.5 in the root mean square (a rounding to bf16 leaves 2^-9.25), and sums in fp32.  y and the pair are then rounded once.
Rounding hides small errors from a tolerance: it is the number of elements that fall on the other side of a rounding which shows them.
An error e in a value whose neighbours are ulp apart moves it to another one with probability |e| / ulp.  DELTA bounds e relative to the
root mean square of its row: an unscaled logit of |q| = |k| = 8 is off by 8 sqrt(2) 2^-18.5 = 2^-15 through x, its weight by that much of
itself, and the output, which averages the weights' errors, by less; the four products behind it add 2^-18.5 each, fp32 sums 2^-20.
Rounding one of the vectors to bf16 instead moves more elements than DELTA can: tests/test_paged_step_precision.py plants that, one
vector at a time, and finds head and remainder at 2^-17."""
from __future__ import annotations

import numpy as np

from paper_2604_21215_amd import inputs as gen
from tests import paged_ref as ref

DELTA = 2.0 ** -15
VECTORS = ("x", "q", "k_t", "v_t", "a", "h", "u", "z")   # in the order in which a step makes them


def _few(S, *front, most=60):
    """Positions: those given, then short ones."""
    return list(front) + [(7 * s) % most for s in range(S - len(front))]


# name, dtype, bits, d, F, max_pos, page, alibi, scale, positions, (wavefronts, parts) of its attention, which products, tiles of W1's workgroups
# positions: -1 idle, max_pos + 1 beyond the bound
FORMS = [
    # the join of parts, on the products of few rows, of 8 to 65536 / d, and of many
    ("join_few", "bf16", 0, 256, 512, 3000, 16, 0.0, 1.0, [3000, 0, -1, 3001, 1500], (4, 12), "mm", None),
    ("join_few_8bit", "bf16", 8, 256, 512, 3000, 32, 8.0, 0.125, [3000, 0, -1, 3001, 1500], (4, 12), "mm", None),
    ("join_own", "bf16", 8, 256, 512, 3000, 64, 0.0, 1.0, _few(9, 3000, 0, -1, 3001, 1025), (4, 12), "own", 1),
    ("join_wide", "bf16", 0, 512, 512, 2100, 64, 8.0, 0.125, _few(140, 2100, 0, -1, 2101, 1500, 1056), (4, 2), "mm", None),
    ("join_wide_8bit", "bf16", 8, 512, 1024, 2100, 32, 0.0, 1.0, _few(140, 2100, 0, -1, 2101, 1500, 1056), (4, 2), "mm", None),
    ("join_f32", "f32", 0, 128, 512, 3000, 16, 8.0, 1.0, [3000, 0, -1, 3001, 1500], (4, 12), "own", 1),
    ("join_f32_8bit", "f32", 8, 128, 264, 3000, 256, 0.0, 0.125, [2999, 0, -1, 3001, 256], (4, 12), "own", 1),
    ("join_odd_width", "bf16", 0, 192, 328, 2000, 16, 0.0, 1.0, [2000, 0, -1, 2001], (4, 8), "own", 1),
    # sixteen wavefronts, in one part and in two
    ("sixteen", "bf16", 0, 256, 512, 1000, 16, 8.0, 0.125, [1000, 0, -1, 1001, 999], (16, 1), "mm", None),
    ("sixteen_join", "bf16", 0, 1024, 1024, 16384, 256, 0.0, 0.125, _few(17, 16384, 0, -1, 16385, 9000, 8192), (16, 2), "own", 1),
    # four tiles of outputs a workgroup: one product of five, and all of them
    ("tiles_1024", "bf16", 0, 1024, 4096, 60, 16, 0.0, 1.0, _few(64, 60, 0, -1, 61), (4, 1), "own", 4),
    ("tiles_320", "bf16", 8, 320, 1280, 60, 16, 8.0, 0.125, _few(200, 60, 0, -1, 61), (4, 1), "own", 4),
    ("tiles_all", "bf16", 0, 576, 640, 60, 16, 0.0, 1.0, _few(464, 60, 0, -1, 61), (4, 1), "own", 4),
    ("tiles_all_f32", "f32", 8, 576, 640, 60, 16, 0.0, 0.125, _few(464, 60, 0, -1, 61), (4, 1), "own", 4),
    # the stack engine's products over several tiles of 16 rows
    ("many_tiles", "bf16", 0, 256, 1024, 60, 16, 0.0, 1.0, _few(260, 60, 0, -1, 61), (4, 1), "mm", None),
    ("many_tiles_8bit", "bf16", 8, 256, 768, 60, 16, 8.0, 0.125, _few(261, 60, 0, -1, 61), (4, 1), "mm", None),
    # unscaled logits on the remaining ones
    ("few_rows", "bf16", 0, 512, 2048, 200, 16, 0.0, 1.0, [200, 0, -1, 63, 64], (4, 1), "mm", None),
    ("one_row", "bf16", 0, 1024, 2048, 100, 16, 0.0, 1.0, [100], (4, 1), "mm", None),
    ("wide", "bf16", 0, 512, 2048, 100, 16, 0.0, 1.0, _few(140, 100, 0, -1), (4, 1), "mm", None),
    ("own", "bf16", 0, 512, 1024, 100, 16, 0.0, 1.0, _few(33, 100, 0, -1), (4, 1), "own", 1),
]
NAMES = [f[0] for f in FORMS]


def inputs(form, seed=1):
    """x, weights, gains.  x is small against what the layer adds to it (its norm takes its size away): y shows the branches."""
    _, dtype, _, d, F, _, _, _, _, pos = form[:10]
    rng = np.random.default_rng(seed + d + len(pos))
    x = (rng.standard_normal((len(pos), d)) * 0.05).astype(np.float32)
    if dtype == "bf16":
        x = gen.round_to_bf16(x)
    return x, gen.make_layer_weights(31, 0, d, F, dtype), gen.random_gains(31, d, dtype)


def step(w, g, x, caches, H, scale, alibi, alpha=1.0, eps=1e-6, alter=lambda name, u: u):
    """The layer's step in float64 (rows x [S, d], caches (K, V) [n, H, 64] of each) -> y, k, v before their rounding.  alter(name, u) changes
    a vector on its way into the next product."""
    from scipy.special import erf
    S, d = x.shape
    head = lambda u, gg: ref.rms(u.reshape(S, H, 64), gg.reshape(H, 64), eps)  # noqa: E731
    n = alter("x", ref.rms(x, g["g_attn"], eps))
    q, kt = alter("q", head(n @ w["Wq"].T, g["g_q"])), alter("k_t", head(n @ w["Wk"].T, g["g_k"]))
    vt = alter("v_t", (n @ w["Wv"].T).reshape(S, H, 64))
    a = alter("a", np.stack([ref.attention(q[s], *caches[s], kt[s], vt[s], scale, alibi, 0.0)[0] for s in range(S)]).reshape(S, d))
    h = x + alpha * a @ w["Wo"].T
    u = alter("h", ref.rms(h, g["g_mlp"], eps)) @ w["W1"].T
    z = h + alpha * alter("u", 0.5 * u * (1 + erf(u / np.sqrt(2.0)))) @ w["W2"].T
    m = alter("z", ref.rms(z, g["g_kv"], eps))
    return z, head(m @ w["Wk"].T, g["g_k"]), (m @ w["Wv"].T).reshape(S, H, 64)


def bf16_ulp(u):
    """Distance of the bf16 numbers around u (normal ones)."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(u), 2.0 ** -126))) - 7)


def to_bf16(u):
    ulp = bf16_ulp(u)
    return np.rint(u / ulp) * ulp


def row_step(u):
    """The step of each 8-bit row of u [..., 64], [..., 1]."""
    _, byte = ref.quantise(u)
    return np.exp2(byte.astype(np.float64) - 127)[..., None]


def moved(got, want, spacing):
    """(elements of got that are another multiple of their spacing than want rounds to, how many the errors of DELTA may move)."""
    flips = np.abs(got - np.rint(want / spacing) * spacing) > 0.25 * spacing
    rms = np.sqrt((want ** 2).mean(-1, keepdims=True))
    expected = np.minimum(1.0, DELTA * rms / spacing * np.ones_like(want)).sum()
    return int(flips.sum()), expected + 6 * np.sqrt(expected) + 3
