"""What DeviceStack and PagedCaches refuse before a kernel could read past an array, on the CPU with a context that records its calls."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2604_21215_amd.paged import PagedCaches  # noqa: E402
from paper_2604_21215_amd.stack import DeviceStack  # noqa: E402

LAYERS, HEADS, ROWS, CACHED, CAP, VOCAB = 2, 1, 3, 20, 25, 40


def _stack():
    calls = []

    class Context:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, a))

    ds = DeviceStack.__new__(DeviceStack)
    ds.ctx, ds.dtype, ds.device, ds.d, ds.H, ds.vocab = Context(), "f32", "cpu", 64 * HEADS, HEADS, VOCAB
    ds.layers = [SimpleNamespace(struct=None)] * LAYERS
    ds.embedding = ds.lm_head = torch.zeros((VOCAB, 64 * HEADS))
    ds.g_final = ds.head4 = ds.K = ds.V = None
    return ds, calls


def _prefilled(ds):
    ds.K = [torch.zeros((CAP, ROWS, HEADS, 64)) for _ in range(LAYERS)]
    ds.V = [torch.zeros_like(k) for k in ds.K]


def _caches(places=ROWS, layers=LAYERS, **kw):
    return PagedCaches(layers, HEADS, places, 64, 12, page_len=16, dtype="f32", device="cpu", **kw)


@pytest.mark.parametrize("lens", [[4, 4], [4, 4, 4, 4], [4, CAP + 1, 4], [64, 0, 0]])
def test_into_pages_refuses(lens):
    ds, calls = _stack()
    _prefilled(ds)
    c = _caches(places=4)
    with pytest.raises(ValueError):
        ds.into_pages(c, lens)
    assert not calls and len(c.free) == 12


def test_into_pages_refuses_without_a_prefill_and_other_caches():
    ds, calls = _stack()
    with pytest.raises(ValueError):
        ds.into_pages(_caches(), [1, 1, 1])
    _prefilled(ds)
    for c in (_caches(places=2), _caches(layers=LAYERS - 1)):
        with pytest.raises(ValueError):
            ds.into_pages(c, [1, 1, 1])
        assert len(c.free) == 12
    assert not calls
    c = _caches(places=5)            # more places than rows of the prefill is fine
    ds.into_pages(c, iter([CACHED, -1, 0]))
    assert c.held == [2, 0, 1, 0, 0] and [n for n, _ in calls] == ["rt_cache_write"] * LAYERS


def test_decode_step_paged_refuses():
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    ds, calls = _stack()
    c = _caches()
    ds.decode_step_paged(c, i32(1, 2, 3), i32(0, -1, 4), 5)
    assert [n for n, _ in calls] == ["rt_embed_rows"] + ["rt_decode_step_paged"] * LAYERS + ["rt_lm_head"]
    del calls[:]
    for caches, ids, pos in ((c, i32(1, 2, 3, 4), i32(0, 0, 0, 0)), (c, i32(1, 2, 3), i32(0, 0)), (c, i32(1, 2, 3).long(), i32(0, 0, 0)),
                             (c, i32(1, 2, 3), i32(0, 0, 0).long()), (c, i32(1, 2, 3), i32(0, 9, 0, 9, 0, 9)[::2]),
                             (c, i32(1, 9, 2, 9, 3, 9)[::2], i32(0, 0, 0)), (c, i32(1, 2, 3).view(3, 1), i32(0, 0, 0)),
                             (c, i32(1, 2, 3), torch.zeros(3, dtype=torch.int32, device="meta")), (_caches(layers=LAYERS + 1), i32(1, 2, 3), i32(0, 0, 0))):
        with pytest.raises(ValueError):
            ds.decode_step_paged(caches, ids, pos, 5)
    with pytest.raises(ValueError):     # no packed weights
        ds.decode_step_paged(c, i32(1, 2, 3), i32(0, 0, 0), 5, head4=True)
    assert not calls


def test_reserve_refuses_what_is_no_place_and_checks_an_iterator():
    c = _caches()
    for lengths in ([1, 1, 1, 1], iter([65, 0, 0]), iter([1, 1, 1, 1])):
        with pytest.raises(ValueError):
            c.reserve(lengths)
        assert c.held == [0, 0, 0] and len(c.free) == 12
    c.reserve(iter([17, 0]))            # the places that are not named keep what they hold
    assert c.held == [2, 0, 0]
    for place in (-1, 3):
        with pytest.raises(ValueError):
            c.release(place)
    assert c.held == [2, 0, 0]
