"""Equal decoding steps give equal bits: steps of few rows at widths where a row's sum of squares comes from several wavefronts, from
pages and over the contiguous cache, called again and again and replayed from a graph."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
REPEATS = 30


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")


def _ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _layer(seed, d):
    from paper_2604_21215_amd import torch_io as tio
    return tio.DeviceLayer(gen.make_layer_weights(seed, 0, d, 4 * d, "bf16"), gen.random_gains(seed, d, "bf16"), "bf16")


@pytest.mark.parametrize("d,S,bits", [(512, 1, 0), (512, 7, 8), (1024, 1, 0), (1024, 5, 0), (1024, 5, 8), (1280, 3, 0)])
def test_steps_from_pages_repeat(d, S, bits):
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(d + S)
    H, pos = d // 64, [90, 40, 0, 17, 64, 3, 89][:S]
    pool = ref.Pool(rng, "bf16", bits, S, H, pos, 16, room=1)
    dl = _layer(5, d)
    st = torch.cuda.Stream()
    ctx = binding.RTContext(d, H, 4 * d, S, 1, "bf16", rms_eps=1e-6, stream=st.cuda_stream, reserve=binding.RT_RESERVE_PAGED)
    try:
        x, at = torch.randn((S, d), device="cuda:0").bfloat16(), _ints(pos)
        y, (ko, vo) = torch.zeros_like(x), (torch.zeros((S, 1, H, 64), device="cuda:0").bfloat16() for _ in range(2))

        def step():
            ctx.rt_decode_step_paged(dl.struct, pool.cache(), x, at, 90, y)
            ctx.rt_cache_read(pool.cache(), at, None, ko, vo)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        first = None
        for rep in range(2 * REPEATS):
            for t in (y, ko, vo):
                t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(st):
                graph.replay() if rep % 2 else step()
            torch.cuda.synchronize()
            now = [t.clone() for t in (y, ko, vo)]
            first = first or now
            assert float(now[0].float().abs().max()) > 0
            for a, b in zip(now, first):
                assert torch.equal(a, b), rep
    finally:
        ctx.rt_destroy()


def test_steps_over_the_contiguous_cache_repeat():
    """The same products serve rt_decode_step where it runs as launches."""
    from paper_2604_21215_amd import binding
    d, B, N = 1024, 5, 40
    H, dl = d // 64, _layer(6, 1024)
    ctx = binding.RTContext(d, H, 4 * d, B, N, "bf16", rms_eps=1e-6, flags=binding.RT_FLAG_ENGINE_STEPWISE,
                            stream=torch.cuda.current_stream().cuda_stream)
    try:
        x = torch.randn((B, d), device="cuda:0").bfloat16()
        K = torch.randn((N, B, H, 64), device="cuda:0").bfloat16()
        V, y, first = torch.randn_like(K), torch.zeros_like(x), None
        for rep in range(REPEATS):
            ctx.rt_decode_step(dl.struct, x, N - 1, y, K, V)
            torch.cuda.synchronize()
            now = [t.clone() for t in (y, K, V)]
            first = first or now
            for a, b in zip(now, first):
                assert torch.equal(a, b), rep
    finally:
        ctx.rt_destroy()
