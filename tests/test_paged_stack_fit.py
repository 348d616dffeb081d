"""DeviceStack takes caches of its own heads, type and device only, on the CPU with a context that records its calls."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2604_21215_amd.paged import PagedCaches  # noqa: E402
from paper_2604_21215_amd.stack import DeviceStack  # noqa: E402

LAYERS, ROWS, MOST = 2, 3, 64


def _stack(heads, dtype, cap=25):
    calls = []

    class Context:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a))

    ds = DeviceStack.__new__(DeviceStack)
    ds.ctx, ds.dtype, ds.device, ds.d, ds.H, ds.vocab = Context(), dtype, "cpu", 64 * heads, heads, 40
    ds.layers = [SimpleNamespace(struct=None)] * LAYERS
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    ds.embedding = ds.lm_head = torch.zeros((40, 64 * heads), dtype=td)
    ds.g_final = ds.head4 = None
    ds.K = [torch.zeros((cap, ROWS, heads, 64), dtype=td) for _ in range(LAYERS)]
    ds.V = [torch.zeros_like(k) for k in ds.K]
    return ds, calls


def _both(ds, c):
    ds.into_pages(c, [4, 0, 9])
    ids, pos = torch.zeros(ROWS, dtype=torch.int32), torch.zeros(ROWS, dtype=torch.int32)
    ds.decode_step_paged(c, ids, pos, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [0, 8])
def test_other_caches_are_refused(dtype, bits):
    other = "bf16" if dtype == "f32" else "f32"
    make = lambda heads, dt: PagedCaches(LAYERS, heads, ROWS, MOST, 12, page_len=16, bits=bits, dtype=dt, device="cpu")  # noqa: E731
    ds, calls = _stack(2, dtype)
    _both(ds, make(2, dtype))
    assert len(calls) == 2 * LAYERS + 2
    del calls[:]
    wrong = [make(1, dtype), make(3, dtype), make(4, other)] + ([] if bits else [make(2, other)])
    for c in wrong:
        ids, pos = torch.zeros(ROWS, dtype=torch.int32), torch.zeros(ROWS, dtype=torch.int32)
        with pytest.raises(ValueError, match="heads"):
            ds.into_pages(c, [4, 0, 9])
        with pytest.raises(ValueError, match="heads"):
            ds.decode_step_paged(c, ids, pos, 5)
        assert len(c.free) == 12
    if bits:        # codes are codes: the type that a cache of 8 bits was made with does not matter
        _both(ds, make(2, other))
        del calls[:]
    c = make(2, dtype)
    c.table = c.table.to("meta")
    with pytest.raises(ValueError, match="meta"):
        ds.into_pages(c, [4, 0, 9])
    assert not calls


def test_a_sequence_that_fills_its_place_moves_into_pages():
    ds, calls = _stack(2, "bf16", cap=MOST + 6)
    c = PagedCaches(LAYERS, 2, ROWS, MOST, 12, page_len=16, dtype="bf16", device="cpu")
    ds.into_pages(c, [MOST, MOST - 1, 0])
    assert c.held == [4, 4, 1] and [n for n, _ in calls] == ["rt_cache_write"] * LAYERS
    c = PagedCaches(LAYERS, 2, ROWS, MOST, 12, page_len=16, dtype="bf16", device="cpu")
    with pytest.raises(ValueError):
        ds.into_pages(c, [MOST + 1, 0, 0])
    assert len(c.free) == 12 and len(calls) == LAYERS
