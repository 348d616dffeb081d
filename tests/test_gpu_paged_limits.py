"""The paged cache's operators at the ends of their ranges."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")


def _ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _context(d, rows, dtype, **kw):
    from paper_2604_21215_amd import binding
    return binding.RTContext(d, d // 64, kw.pop("F", 4 * d), rows, 1, dtype, rms_eps=1e-6, stream=torch.cuda.current_stream().cuda_stream, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_next_to_the_largest_number_stay_finite(dtype):
    """In 8 bits, values past 63.5 2^122 read as 63 2^122; the other values of their row are off by half of 2^122; and an attention over such
    keys (weighted by a query of zeros) and finite values is finite."""
    from paper_2604_21215_amd import torch_io as tio
    rng = np.random.default_rng(1)
    top = np.finfo(np.float32).max if dtype == "f32" else gen.round_to_bf16(np.array([3.3895e38], dtype=np.float32))[0]
    u = (rng.uniform(-1, 1, (1, 40, 1, 64)) * top).astype(np.float32)
    u[0, :, 0, 5], u[0, ::3, 0, 9] = top, -top
    if dtype == "bf16":
        u = gen.round_to_bf16(u)
    pool = ref.Pool(rng, dtype, 8, 1, 1, [40], 16)
    ctx = _context(64, 1, dtype)
    try:
        k = tio.to_device(u, dtype)
        v = tio.to_device(gen.round_to_bf16((u / top).astype(np.float32)), dtype)
        ko, vo, q = torch.zeros_like(k), torch.zeros_like(v), torch.zeros((1, 1, 64), dtype=k.dtype, device="cuda:0")
        out = torch.zeros_like(q)
        ctx.rt_cache_write(pool.cache(), _ints([0]), None, k, v)
        ctx.rt_cache_read(pool.cache(), _ints([0]), None, ko, vo)
        ctx.rt_paged_attention(pool.cache(), _ints([40]), 40, q, None, None, out)
        torch.cuda.synchronize()
        got = tio.to_host(ko)[0, :, 0]
        assert bool(torch.isfinite(out).all())
    finally:
        ctx.rt_destroy()
    w, step = u[0, :, 0].astype(np.float64), 2.0 ** 122
    want = np.clip(np.rint(w / step), -63, 63) * step
    np.testing.assert_array_equal(got, want)
