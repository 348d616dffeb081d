"""The paged cache's arithmetic (exponents of 8-bit rows, places of rows, how a call is cut into splits) and the refusals of its entry
points, on the CPU: the headers are compiled by themselves (paged_args_check.cpp).  And the host packer of 4-bit weights."""
import os
import subprocess

import numpy as np
import pytest

from paper_2604_21215_amd import binding, inputs as gen

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_21215_amd", "csrc")
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paged_args") / "check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "paged_args_check.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("check", ["exponents", "rows", "plans", "refusals"])
def test_paged_args(program, check):
    r = subprocess.run([program, check], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def mx4_values(codes, exps):
    """What packed weights stand for, float64 [rows, cols]."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)
    v = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    return v * np.exp2(exps.astype(np.float64) - 127).repeat(32, 1)


def _nearest(u):
    """Nearest element, ties to the even code: by comparison with every element."""
    dist = np.abs(np.abs(u)[..., None] - E2M1)
    best = dist.min(-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])   # even codes first
    return E2M1[order[np.argmax((dist == best)[..., order], -1)]] * np.sign(u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "ties", "small", "spread"])
def test_mx4_pack(dtype, kind):
    rng = np.random.default_rng(7)
    W = {"normal": lambda: rng.standard_normal((37, 96)) * 0.02,
         "ties": lambda: rng.choice([0, .25, .5, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, -.25, -5, 7, 12], (37, 96)),
         "small": lambda: rng.standard_normal((37, 96)) * 2.0 ** -126,
         "spread": lambda: rng.standard_normal((37, 96)) * np.exp2(rng.integers(-120, 120, (37, 1)).astype(float))}[kind]().astype(np.float32)
    W[3, 32:64] = 0.0
    if dtype == "bf16":
        W = gen.round_to_bf16(W)
    codes, exps = binding.rt_mx4_pack(W if dtype == "f32" else gen.f32_to_bf16_bits(W))
    assert exps.min() >= 1 and exps.max() <= 254
    w, got = W.astype(np.float64).reshape(37, 3, 32), mx4_values(codes, exps).reshape(37, 3, 32)
    assert np.all(got[3, 1] == 0)
    top = np.abs(w).max(-1, keepdims=True)
    e = exps.astype(np.float64).reshape(37, 3, 1) - 127
    np.testing.assert_array_equal(got, _nearest(w / np.exp2(e)) * np.exp2(e))
    # the scale: of the smallest that reaches the largest weight and the one below, the one with the smaller error
    reach = np.ceil(np.log2(np.maximum(top, 2.0 ** -200) / 6.0) - 1e-12)
    reach = np.maximum(np.where(6 * np.exp2(reach) < top, reach + 1, reach), -126)
    err = lambda s: ((w - _nearest(w / np.exp2(s)) * np.exp2(s)) ** 2).sum(-1, keepdims=True)  # noqa: E731
    want = np.where((err(reach - 1) < err(reach)) & (reach > -126), reach - 1, reach)
    some = top > 0
    np.testing.assert_array_equal(e[some], want[some])
    # a nearest element is off by at most a third of the value (3/4 lies midway between 1/2 and 1), or half the smallest element
    fits = np.abs(w) <= 6 * np.exp2(e)
    assert np.all(np.abs(w - got)[fits] <= np.maximum(np.abs(w) / 3, np.exp2(e) / 4)[fits])


def test_mx4_pack_refusals():
    L = binding.load()
    W = np.zeros((2, 64), dtype=np.float32)
    codes, exps = np.zeros((2, 32), dtype=np.uint8), np.zeros((2, 2), dtype=np.uint8)
    go = lambda w, dt, r, c, a, b: L.rt_mx4_pack(w, dt, r, c, a, b)  # noqa: E731
    p, a, b = W.ctypes.data, codes.ctypes.data, exps.ctypes.data
    assert go(p, 0, 2, 64, a, b) == binding.RT_OK
    for bad in ((None, 0, 2, 64, a, b), (p, 0, 2, 64, None, b), (p, 0, 2, 64, a, None), (p, 2, 2, 64, a, b), (p, 0, 0, 64, a, b),
                (p, 0, 2, 63, a, b), (p, 0, 2, 0, a, b)):
        assert go(*bad) == binding.RT_ERR_INVALID_ARG
    for v in (np.nan, np.inf, -np.inf):
        W[1, 5] = v
        assert go(p, 0, 2, 64, a, b) == binding.RT_ERR_INVALID_ARG
    with pytest.raises(binding.RTError):
        binding.rt_mx4_pack(np.zeros((2, 48), dtype=np.float32))


def test_entry_points_refuse_a_null_context():
    L = binding.load()
    assert L.rt_cache_write(None, None, 1, None, None, 1, None, None, 0, 0) == binding.RT_ERR_INVALID_ARG
    assert L.rt_cache_read(None, None, 1, None, None, 1, None, None, 0, 0) == binding.RT_ERR_INVALID_ARG
    assert L.rt_paged_attention(None, None, 1, None, 1, None, 64, None, None, 64, None, 64, None) == binding.RT_ERR_INVALID_ARG
    assert L.rt_decode_step_paged(None, None, None, None, 1, None, 1, None) == binding.RT_ERR_INVALID_ARG
    assert L.rt_lm_head_mx4(None, None, None, None, 1, None, 64, 1, None) == binding.RT_ERR_INVALID_ARG
