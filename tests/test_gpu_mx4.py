"""rt_lm_head_mx4 against float64 over the values its packed matrix stands for: both storage types, batch tiles of up to 16 and more,
vocabularies that end inside a tile, widths that end inside a block group, strided rows, scales at both ends, bytes that are no scale."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests.test_paged_args import mx4_values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _run(dtype, codes, exps, g, z, norm_free=False, shift=0):
    """z [B, 3, d]: rows at a stride, the middle ones are read; shift: they start that many elements on, the stride is odd."""
    from paper_2604_21215_amd import binding, torch_io as tio
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    B, _, d = z.shape
    vocab = codes.shape[0]
    ctx = binding.RTContext(d, d // 64, 64, B, 1, dtype, rms_eps=1e-6, flags=binding.RT_FLAG_NORM_FREE if norm_free else 0,
                            stream=torch.cuda.current_stream().cuda_stream)
    try:
        zd = tio.to_device(np.pad(z.reshape(B, 3 * d), ((0, 0), (shift, shift and 1 - shift % 2))), dtype)[:, shift:shift + 3 * d]
        zd = zd.unflatten(1, (3, d))
        out = torch.full((B + 1, vocab), 7.0, dtype=torch.float32, device="cuda:0")
        ctx.rt_lm_head_mx4(torch.from_numpy(codes).to("cuda:0"), torch.from_numpy(exps).to("cuda:0"),
                           None if g is None else tio.to_device(g, dtype), zd[:, 1], zd.stride(0), B, out[:B])
        torch.cuda.synchronize()
        got = out.cpu().numpy().astype(np.float64)
    finally:
        ctx.rt_destroy()
    assert np.all(got[B] == 7)
    return got[:B]


@pytest.mark.parametrize("dtype,d,vocab,B,norm_free,gain", [
    ("bf16", 64, 1, 1, False, True), ("bf16", 128, 15, 16, False, True), ("bf16", 192, 333, 17, False, False), ("bf16", 1024, 2064, 8, False, True),
    ("bf16", 1024, 50, 1, False, True), ("bf16", 512, 4097, 33, True, True), ("f32", 128, 1000, 3, False, True), ("f32", 320, 130, 40, False, True),
    ("f32", 64, 17, 2, True, False), ("bf16", 4096, 70, 5, False, True), ("bf16", 25856, 20, 2, False, True), ("bf16", 1024, 33000, 2, False, True),
    ("bf16", 768, 515, 100, False, True), ("bf16", 2048, 100, 16, False, True), ("bf16", 1536, 300, 40, False, False), ("bf16", 1088, 90, 3, False, True),
    ("bf16", 3136, 100, 20, False, False), ("bf16", 576, 3000, 64, False, False), ("f32", 1024, 200, 20, False, True), ("f32", 1600, 70, 2, False, True),
    ("f32", 2112, 70, 18, False, False), ("bf16", 4160, 33, 1, True, True), ("bf16", 128, 20000, 65, False, True)])
def test_lm_head_mx4(dtype, d, vocab, B, norm_free, gain):
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(d + vocab + B)
    W = (rng.standard_normal((vocab, d)) * 0.05 * np.exp2(rng.integers(-6, 6, (vocab, 1)).astype(float))).astype(np.float32)
    codes, exps = binding.rt_mx4_pack(W)
    g = rng.uniform(0.5, 1.5, d).astype(np.float32) if gain else None
    z = rng.standard_normal((B, 3, d)).astype(np.float32)
    if dtype == "bf16":
        z, g = gen.round_to_bf16(z), None if g is None else gen.round_to_bf16(g)
    got = _run(dtype, codes, exps, g, z, norm_free)
    z64 = z[:, 1].astype(np.float64)
    n = z64 if norm_free else z64 / np.sqrt((z64 ** 2).mean(-1, keepdims=True) + 1e-6) * (1.0 if g is None else g.astype(np.float64))
    W4 = mx4_values(codes, exps)
    ref = n @ W4.T
    # fp32 operands and sums: a row's elements carry three roundings of 2^-24 and the sum of squares (d additions in 64 lanes) its own;
    # the logit's sums round at 2^-24 of partial sums, which grow like the root of their d terms
    bound = (8 * np.sqrt(d) + d / 64) * 2.0 ** -24 * (np.abs(n) @ np.abs(W4).T)
    err = np.abs(got - ref)
    assert np.all(err <= bound), (err / np.maximum(bound, 1e-300)).max()
    # norm-wise: the rows' three roundings, the two of 1 / rms (common to a row) and the last sums are 2^-22 at most; each of four running
    # sums rounds d / 128 times at up to half of 2^-24 of itself, at random.  Rows rounded to bf16 would be off by 2^-9 / sqrt(3).
    assert np.linalg.norm(got - ref) <= (2.0 ** -22 + 2.0 ** -25 * np.sqrt(d / 128)) * np.linalg.norm(ref)


@pytest.mark.parametrize("dtype,d,B", [("bf16", 1024, 3), ("f32", 128, 17), ("bf16", 64, 1)])
def test_rows_off_16_bytes(dtype, d, B):
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(B)
    codes, exps = binding.rt_mx4_pack((rng.standard_normal((77, d)) * 0.05).astype(np.float32))
    g, z = rng.uniform(0.5, 1.5, d).astype(np.float32), rng.standard_normal((B, 3, d)).astype(np.float32)
    if dtype == "bf16":
        g, z = gen.round_to_bf16(g), gen.round_to_bf16(z)
    a, b = _run(dtype, codes, exps, g, z), _run(dtype, codes, exps, g, z, shift=3)
    n = z[:, 1].astype(np.float64) / np.sqrt((z[:, 1].astype(np.float64) ** 2).mean(-1, keepdims=True) + 1e-6) * g.astype(np.float64)
    bound = (8 * np.sqrt(d) + d / 64) * 2.0 ** -24 * (np.abs(n) @ np.abs(mx4_values(codes, exps)).T)
    assert np.all(np.abs(a - b) <= 2 * bound) and np.all(np.abs(b - n @ mx4_values(codes, exps).T) <= bound)


def test_every_code_and_scale():
    """One row per scale byte, every code in it; the input picks one element: what the matrix stands for, exactly."""
    d, rows = 64, 256
    codes = np.tile(np.arange(16, dtype=np.uint8), (rows, 4)).reshape(rows, 32, 2)
    codes = (codes[..., 0] | (codes[..., 1] << 4)).astype(np.uint8)
    exps = np.stack((np.arange(256), 255 - np.arange(256)), 1).astype(np.uint8)
    with np.errstate(over="ignore"):
        W = mx4_values(codes, np.clip(exps, 1, 254))
    z = np.zeros((16, 3, d), dtype=np.float32)
    for b in range(16):
        z[b, 1, (5 * b) % 64] = 1.0
    got = _run("bf16", codes, exps, None, z, norm_free=True)
    for b in range(16):
        k = (5 * b) % 64
        for r in range(rows):
            # one of the row's blocks has no scale; or holds 4 2^126, 2 2^127 ..: infinities in fp32, and times the other zeros NaN
            if r in (0, 255) or np.abs(W[r]).max() >= 2.0 ** 128:
                assert np.isnan(got[b, r])
            else:
                want = np.float64(np.float32(W[r, k]))
                assert got[b, r] == want or (abs(want) < 2.0 ** -125 and abs(got[b, r] - want) <= 2.0 ** -127), (b, r, got[b, r], want)


def test_rows_that_are_not_finite():
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(1)
    codes, exps = binding.rt_mx4_pack((rng.standard_normal((40, 128)) * 0.05).astype(np.float32))
    z = rng.standard_normal((4, 3, 128)).astype(np.float32)
    z[1, 1, 100] = np.nan
    z[2, 1, 3] = np.inf
    got = _run("f32", codes, exps, None, z)
    assert np.all(np.isnan(got[1])) and np.all(np.isnan(got[2])) and np.all(np.isfinite(got[[0, 3]]))
    free = _run("f32", codes, exps, None, z, norm_free=True)
    with np.errstate(invalid="ignore"):
        want = z[2, 1].astype(np.float64) @ mx4_values(codes, exps).T      # an infinity with its weight's sign, NaN where the weight is 0
    np.testing.assert_array_equal(np.isnan(free[2]), np.isnan(want))
    np.testing.assert_array_equal(np.sign(free[2][~np.isnan(want)]), np.sign(want[~np.isnan(want)]))


@pytest.mark.parametrize("dtype,d,B", [("bf16", 1024, 1), ("bf16", 512, 64), ("f32", 4224, 2)])
def test_captured(dtype, d, B):
    """A captured read-out, replayed on other rows among eager calls: every replay gives the eager call's bits."""
    from paper_2604_21215_amd import binding, torch_io as tio
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    rng = np.random.default_rng(d)
    codes, exps = (torch.from_numpy(a).to("cuda:0") for a in binding.rt_mx4_pack((rng.standard_normal((500, d)) * 0.05).astype(np.float32)))
    st = torch.cuda.Stream()
    ctx = binding.RTContext(d, d // 64, 64, B, 1, dtype, rms_eps=1e-6, stream=st.cuda_stream)
    try:
        z, g = torch.zeros((B, d), dtype=tio.torch_dtype(dtype), device="cuda:0"), torch.ones(d, dtype=tio.torch_dtype(dtype), device="cuda:0")
        out = torch.zeros((B, 500), device="cuda:0")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.rt_lm_head_mx4(codes, exps, g, z, d, B, out)
        for rep in range(3):
            z.copy_(torch.randn((B, d), device="cuda:0"))
            torch.cuda.synchronize()
            with torch.cuda.stream(st):
                ctx.rt_lm_head_mx4(codes, exps, g, z, d, B, out)
            torch.cuda.synchronize()
            eager = out.clone()
            out.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(st):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager) and float(out.abs().max()) > 0
    finally:
        ctx.rt_destroy()
