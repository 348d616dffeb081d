"""The paged cache, the attention of one new token over it and the decoding step from pages, against plain float64 forms: every storage
type and cache width, lengths from none to long ones, pages that end inside a tile, idle places, rows that hold NaN behind the last
position, wrong entries of the page table, non-finite values, strides, captured calls, streams, and the refusals."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")


def _context(d, rows, dtype, **kw):
    from paper_2604_21215_amd import binding
    kw.setdefault("stream", torch.cuda.current_stream().cuda_stream)
    kw.setdefault("rms_eps", 1e-6)
    return binding.RTContext(d, d // 64, kw.pop("F", 4 * d), rows, 1, dtype, **kw)


def _rows(rng, dtype, *shape, std=1.0):
    a = (rng.standard_normal(shape) * std).astype(np.float32)
    return gen.round_to_bf16(a) if dtype == "bf16" else a


def _ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _host(t):
    from paper_2604_21215_amd import torch_io as tio
    return tio.to_host(t)


def _lens(rng, S, most):
    n = rng.integers(0, most + 1, S)
    n[0] = most
    for i, v in enumerate((0, -1, 1, min(most, 63), min(most, 64), min(most, 65))):
        if S > i + 1:
            n[i + 1] = v if v <= most else most
    return n


ATTENTION = [("bf16", 0, 1, 1, 0, 16, 0.0, 1.0, True), ("bf16", 0, 1, 8, 1, 16, 0.0, 1.0, False), ("bf16", 0, 1, 8, 37, 16, 0.0, 1.0, True),
             ("bf16", 0, 9, 5, 300, 16, 8.0, 0.125, True), ("bf16", 8, 9, 5, 300, 16, 8.0, 0.125, True), ("f32", 0, 9, 3, 300, 32, 8.0, 0.125, True),
             ("f32", 8, 9, 3, 513, 64, 0.0, 0.125, False), ("bf16", 8, 3, 16, 2049, 256, 0.0, 1.0, True), ("bf16", 0, 3, 16, 2049, 1024, 8.0, 1.0, False),
             ("f32", 0, 2, 2, 5000, 16, 0.0, 1.0, True), ("bf16", 0, 2, 2, 20011, 64, 0.0, 0.125, True), ("bf16", 8, 2, 2, 20011, 128, 8.0, 0.125, True),
             ("bf16", 8, 70, 2, 130, 32, 0.0, 1.0, True), ("f32", 0, 70, 1, 64, 16, 8.0, 1.0, False), ("bf16", 0, 20, 8, 1500, 64, 8.0, 0.125, True),
             ("bf16", 8, 20, 8, 1300, 16, 0.0, 0.125, False), ("f32", 0, 40, 4, 700, 32, 0.0, 0.125, True), ("bf16", 0, 150, 2, 3200, 128, 0.0, 0.125, True),
             ("f32", 8, 3, 2, 1281, 16, 8.0, 0.125, True), ("bf16", 8, 2, 1, 257, 16, 0.0, 1.0, False)]


@pytest.mark.parametrize("dtype,bits,S,H,most,page,alibi,scale,pair", ATTENTION)
def test_attention(dtype, bits, S, H, most, page, alibi, scale, pair):
    from paper_2604_21215_amd import torch_io as tio
    rng = np.random.default_rng(S * 1000 + most + H)
    lens, d = _lens(rng, S, most), 64 * H
    pool = ref.Pool(rng, dtype, bits, S, H, lens, page)
    # rows of q, the pair and the output lie apart (in the same order of magnitude as in a [q | k | v] tensor)
    qkv = _rows(rng, dtype, S, 3 * d + 64)
    dev = tio.to_device(qkv, dtype)
    q, k_t, v_t = dev[:, :d], dev[:, d:2 * d], dev[:, 2 * d:3 * d]
    out = torch.full((S + 1, d + 8), 7.0, dtype=dev.dtype, device="cuda:0")
    lse = torch.full((S + 1, H), 7.0, device="cuda:0")
    ctx = _context(d, S, dtype, attn_scale=scale, alibi_max_bias=alibi)
    try:
        before = pool.bits_of()
        table = pool.table if (pool.table.shape[1] * page >= most) else None
        assert table is not None
        ctx.rt_paged_attention(pool.cache(), _ints(lens), most, q, k_t if pair else None, v_t if pair else None, out[:S, :d], lse)
        torch.cuda.synchronize()
        got, got_lse = _host(out), _host(lse)
        again, lse2 = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
        ctx.rt_paged_attention(pool.cache(), _ints(lens), most, q, k_t if pair else None, v_t if pair else None, again[:S, :d], lse2)
        torch.cuda.synchronize()
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    finally:
        ctx.rt_destroy()
    for a, b in zip(before, pool.bits_of()):
        np.testing.assert_array_equal(a, b)
    assert np.all(got[S] == 7) and np.all(got[:, d:] == 7) and np.all(got_lse[S] == 7)
    x = qkv.astype(np.float64)
    for s in range(S):
        if lens[s] < 0:
            assert np.all(got[s] == 7) and np.all(got_lse[s] == 7)
            continue
        row = lambda i: x[s, i * d:(i + 1) * d].reshape(H, 64)  # noqa: E731
        o, l, bound, lbound = ref.attention(row(0), pool.K[s], pool.V[s], row(1) if pair else None, row(2) if pair else None, scale, alibi,
                                            HALF[dtype])
        if lens[s] == 0 and not pair:
            assert np.all(got[s, :d] == 0) and np.all(got_lse[s] == -np.inf)
            continue
        err = np.abs(got[s, :d].reshape(H, 64) - o)
        assert np.all(err <= bound), (s, lens[s], (err / bound).max())
        assert np.all(np.abs(got_lse[s] - l) <= lbound), (s, lens[s])


def test_attention_without_lse_on_its_own_stream():
    """A context on a stream of its own: its work is ordered there, the outputs are read after that stream."""
    rng = np.random.default_rng(5)
    lens = [100, 3]
    pool = ref.Pool(rng, "bf16", 0, 2, 4, lens, 16)
    q = torch.randn((2, 4, 64), device="cuda:0").bfloat16()
    n = _ints(lens)
    st = torch.cuda.Stream()
    main = _context(256, 2, "bf16")
    side = _context(256, 2, "bf16", stream=st.cuda_stream)
    try:
        a, b = torch.zeros_like(q), torch.zeros_like(q)
        torch.cuda.synchronize()
        main.rt_paged_attention(pool.cache(), n, 100, q, None, None, a)
        with torch.cuda.stream(st):
            side.rt_paged_attention(pool.cache(), n, 100, q, None, None, b)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and float(a.float().abs().max()) > 0
    finally:
        main.rt_destroy()
        side.rt_destroy()


@pytest.mark.parametrize("bits", [0, 8])
@pytest.mark.parametrize("most", [200, 3000])
def test_wrong_pages_and_lengths_give_nan_rows(bits, most):
    """An entry that names no page, first, in the middle and last; a length beyond max_len: those rows are NaN, the others as without."""
    rng = np.random.default_rng(9)
    S, H = 6, 2
    lens = [most, most, most, most - 1, most, 40]
    pool = ref.Pool(rng, "bf16", bits, S, H, lens, 16)
    q = torch.randn((S, H, 64), device="cuda:0").bfloat16()
    ctx = _context(64 * H, S, "bf16", attn_scale=0.125)
    try:
        fine, lse0 = torch.zeros_like(q), torch.zeros((S, H), device="cuda:0")
        ctx.rt_paged_attention(pool.cache(), _ints(lens), most, q, None, None, fine, lse0)
        last = (most - 1) // 16
        pool.table[1, 0], pool.table[2, last // 2], pool.table[4, last] = -1, pool.Kd.shape[0], 2 ** 31 - 1
        out, lse = torch.zeros_like(q), torch.zeros_like(lse0)
        ctx.rt_paged_attention(pool.cache(), _ints(lens[:5] + [most + 1]), most, q, None, None, out, lse)
        torch.cuda.synchronize()
        for s in range(S):
            if s in (1, 2, 4, 5):
                assert bool(torch.isnan(out[s]).all()) and bool(torch.isnan(lse[s]).all())
            else:
                assert torch.equal(out[s], fine[s]) and torch.equal(lse[s], lse0[s])
    finally:
        ctx.rt_destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(dtype):
    """An infinite value has the weight of its key; a key of minus infinities against a positive query has no weight, and a row of
    nothing else is empty; NaN in a cached row makes the row NaN."""
    from paper_2604_21215_amd import torch_io as tio
    rng = np.random.default_rng(3)
    lens = [70, 70, 70, 5]
    pool = ref.Pool(rng, dtype, 0, 4, 1, lens, 16)
    tab = pool.table.cpu().numpy()
    at = lambda s, p: (int(tab[s, p // 16]), 0, p % 16)  # noqa: E731
    pool.Vd[at(0, 66)][3] = float("inf")
    pool.Kd[at(1, 10)][:] = float("-inf")
    pool.Kd[at(2, 69)][7] = float("nan")
    for p in range(5):
        pool.Kd[at(3, p)][:] = float("-inf")
    q = np.abs(_rows(rng, dtype, 4, 1, 64)) + np.float32(0.25)
    if dtype == "bf16":
        q = gen.round_to_bf16(q)
    ctx = _context(64, 4, dtype, attn_scale=0.125)
    try:
        qd = tio.to_device(q, dtype)
        out, lse = torch.zeros_like(qd), torch.zeros((4, 1), device="cuda:0")
        ctx.rt_paged_attention(pool.cache(), _ints(lens), 70, qd, None, None, out, lse)
        torch.cuda.synchronize()
        got, l = _host(out), _host(lse)
    finally:
        ctx.rt_destroy()
    q64 = q.astype(np.float64)
    o, _, bound, _ = ref.attention(q64[0], pool.K[0], pool.V[0], None, None, 0.125, 0.0, HALF[dtype])
    assert got[0, 0, 3] == np.inf
    keep = np.arange(64) != 3
    assert np.all(np.abs(got[0] - o)[:, keep] <= bound[:, keep])
    rest = np.arange(70) != 10
    o, _, bound, _ = ref.attention(q64[1], pool.K[1][rest], pool.V[1][rest], None, None, 0.125, 0.0, HALF[dtype])
    assert np.all(np.abs(got[1] - o) <= bound)
    assert np.all(np.isnan(got[2])) and np.isnan(l[2, 0])
    assert np.all(got[3] == 0) and l[3, 0] == -np.inf


CACHE = [("bf16", 8, 1, 1, 1, 16), ("bf16", 8, 5, 1, 3, 64), ("bf16", 8, 4, 77, 16, 32), ("f32", 8, 4, 77, 3, 16), ("bf16", 0, 4, 77, 3, 16),
         ("f32", 0, 3, 8, 1, 128), ("f32", 8, 6, 7, 2, 1024), ("bf16", 8, 3, 300, 5, 256)]


@pytest.mark.parametrize("dtype,bits,S,N,H,page", CACHE)
@pytest.mark.parametrize("layout", ["position first", "sequence first", "interleaved"])
def test_cache_write_and_read(dtype, bits, S, N, H, page, layout):
    from paper_2604_21215_amd import torch_io as tio
    rng = np.random.default_rng(S + N + H)
    first = rng.integers(0, 2 * page, S)
    count = rng.integers(0, N + 1, S)
    count[0] = N
    if S >= 3:
        first[1], count[2] = -1, 0
    if S >= 4:
        count[3] = N + 5          # cut to N
    if S >= 5:
        first[4], count[4] = 0, -2
    pool = ref.Pool(rng, dtype, bits, S, H, [0 if f < 0 else int(f) + N for f in first], page)
    before = pool.bits_of()
    shape = {"position first": (N, S, H, 64), "sequence first": (S, N, H, 64), "interleaved": (S, N, 2, H, 64)}[layout]
    def view(pair):
        if layout == "position first":
            return tuple(t.transpose(0, 1) for t in pair)
        return pair if layout == "sequence first" else (pair[0][:, :, 0], pair[0][:, :, 1])
    host = [_rows(rng, dtype, *shape, std=10.0 ** float(rng.integers(-3, 3))) for _ in range(2)]
    for h in host:   # rows of zeros, of one large value, of the smallest numbers, at the border of two steps, and not finite
        flat = h.reshape(-1, 64)
        n = flat.shape[0]
        for i, v in enumerate((0.0, 1e30, 1e-42, 127 / 128, np.inf, np.nan, -np.inf, 3e38)):
            if n > 3 * i + 2:
                flat[(3 * i + 2) % n, 5] = v
        if n > 30:
            flat[30] = 0.0
            flat[29] = np.float32(127 / 128) * np.sign(flat[29])
        if dtype == "bf16":
            h.reshape(-1)[:] = np.where(np.isfinite(flat), gen.round_to_bf16(np.where(np.isfinite(flat), flat, 0)), flat).reshape(-1)
    def device(a):   # bits of what is not finite as they are
        t = tio.to_device(np.where(np.isfinite(a), a, 0), dtype)
        for v in (np.inf, -np.inf):
            t[torch.from_numpy(a == v).to("cuda:0")] = v
        t[torch.from_numpy(np.isnan(a)).to("cuda:0")] = float("nan")
        return t
    kd, vd = view([device(h) for h in host])
    ctx = _context(64 * H, 1, dtype)   # S is not bound by max_batch
    try:
        ko, vo = view([torch.full(shape, 7.0, dtype=kd.dtype, device="cuda:0") for _ in range(2)])
        ctx.rt_cache_write(pool.cache(), _ints(first), _ints(count), kd, vd)
        ctx.rt_cache_read(pool.cache(), _ints(first), _ints(count), ko, vo)
        torch.cuda.synchronize()
        got = [_host(t.contiguous()) for t in (ko, vo)]
        rows = [_host(t.contiguous()) for t in (kd, vd)]
    finally:
        ctx.rt_destroy()
    after = pool.bits_of()
    tab, touched = pool.table.cpu().numpy(), np.zeros(after[0].shape[:3], dtype=bool)
    for s in range(S):
        n = min(int(count[s]), N) if first[s] >= 0 else 0
        for i in range(N):
            if i >= n:
                assert all(np.all(g[s, i] == 7) for g in got)
                continue
            p = int(first[s]) + i
            page_of, row = tab[s, p // page], p % page
            touched[page_of, :, row] = True
            for w in range(2):
                u = rows[w][s, i]
                if bits:
                    c, b = ref.quantise(u)
                    np.testing.assert_array_equal(after[2 + w][page_of, :, row], b)
                    np.testing.assert_array_equal(after[w][page_of, :, row].view(np.int8), np.where(b[:, None] == 255, 0, c))
                    u = ref.values(c, b)
                np.testing.assert_array_equal(got[w][s, i], u)
    for a, b in zip(after, before):
        np.testing.assert_array_equal(a[~touched], b[~touched])


def test_cache_rows_without_a_page():
    """Positions past the table and entries that name no page: nothing is written for them, and they read as NaN."""
    rng = np.random.default_rng(1)
    for bits in (0, 8):
        pool = ref.Pool(rng, "bf16", bits, 2, 2, [32, 32], 16)   # two pages each and one entry more, which is wrong
        pool.table[:, 2] = torch.tensor([-5, pool.Kd.shape[0]], dtype=torch.int32)
        pool.table[1, 0] = -1
        before = pool.bits_of()
        k, v = (torch.randn((2, 40, 2, 64), device="cuda:0").bfloat16() for _ in range(2))
        ctx = _context(128, 2, "bf16")
        try:
            first = _ints([30, 12])   # the table ends at position 48
            ctx.rt_cache_write(pool.cache(), first, None, k, v)
            ko, vo = torch.zeros_like(k), torch.zeros_like(v)
            ctx.rt_cache_read(pool.cache(), first, None, ko, vo)
            torch.cuda.synchronize()
        finally:
            ctx.rt_destroy()
        there = {0: [0, 1], 1: list(range(4, 20))}   # rows whose positions have a page
        for s in range(2):
            for i in range(40):
                for src, dst in ((k, ko), (v, vo)):
                    if i in there[s]:
                        assert bool((dst[s, i].float() - src[s, i].float()).abs().max() <= src[s, i].float().abs().max() / 127 if bits
                                    else torch.equal(dst[s, i], src[s, i]))
                    else:
                        assert bool(torch.isnan(dst[s, i]).all())
        changed = sum(int((a != b).reshape(a.shape[0], 2, 16, -1).any(-1).any(1).sum()) for a, b in zip(before[:1], pool.bits_of()[:1]))
        assert changed == 18


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements (8 bits), rows in its last pages."""
    H, page = 32, 64
    pages = 2 ** 32 // (H * page * 64) + 8
    K = torch.empty((pages, H, page, 64), dtype=torch.int8, device="cuda:0")
    V = torch.empty_like(K)
    ke, ve = (torch.empty((pages, H, page), dtype=torch.uint8, device="cuda:0") for _ in range(2))
    from paper_2604_21215_amd import binding
    table = torch.tensor([[pages - 1, 3], [0, pages - 2]], dtype=torch.int32, device="cuda:0")
    cache = binding.make_cache(K, V, table, ke, ve)
    k, v = (torch.randn((2, 100, H, 64), device="cuda:0").bfloat16() for _ in range(2))
    q = torch.randn((2, H, 64), device="cuda:0").bfloat16()
    ctx = _context(64 * H, 2, "bf16", attn_scale=0.125, F=64)
    try:
        zero, lens = _ints([0, 0]), _ints([100, 100])
        ctx.rt_cache_write(cache, zero, None, k, v)
        ko, vo, out = torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(q)
        ctx.rt_cache_read(cache, zero, None, ko, vo)
        ctx.rt_paged_attention(cache, lens, 100, q, None, None, out)
        torch.cuda.synchronize()
        assert bool(((ko.float() - k.float()).abs() <= k.float().abs().amax(-1, keepdim=True) / 127).all())
        k64, v64, q64 = _host(ko), _host(vo), _host(q)
        for s in range(2):
            o, _, bound, _ = ref.attention(q64[s], k64[s], v64[s], None, None, 0.125, 0.0, HALF["bf16"])
            assert np.all(np.abs(_host(out)[s] - o) <= bound)
    finally:
        ctx.rt_destroy()


def _layer(seed, dtype, d, F):
    w = gen.make_layer_weights(seed, 0, d, F, dtype)
    g = gen.random_gains(seed, d, dtype)
    return w, g


STEP = [("bf16", 0, 1, 256, 1024, 0, 16, 0.0, False), ("bf16", 0, 5, 256, 1024, 100, 16, 8.0, False), ("bf16", 8, 5, 512, 2048, 300, 32, 0.0, False),
        ("bf16", 8, 40, 512, 1024, 70, 16, 8.0, False), ("bf16", 0, 33, 512, 1536, 50, 16, 0.0, True), ("bf16", 8, 17, 256, 512, 600, 64, 0.0, True),
        ("bf16", 0, 4, 320, 640, 90, 16, 8.0, False), ("bf16", 8, 11, 192, 768, 90, 16, 0.0, False), ("f32", 0, 4, 128, 512, 130, 16, 8.0, False),
        ("f32", 8, 9, 128, 264, 600, 32, 0.0, True), ("bf16", 8, 7, 256, 1024, 300, 16, 0.0, False), ("bf16", 8, 20, 256, 512, 40, 16, 8.0, False),
        ("bf16", 8, 130, 512, 512, 30, 16, 0.0, False), ("bf16", 0, 140, 512, 2048, 20, 16, 8.0, False), ("bf16", 0, 30, 320, 264, 90, 16, 0.0, True)]


@pytest.mark.parametrize("dtype,bits,S,d,F,most,page,alibi,norm_free", STEP)
def test_decode_step_from_pages(dtype, bits, S, d, F, most, page, alibi, norm_free):
    """y and the new pair against the float64 layer over the values that the cache holds.  Tolerances: norm-wise those of the other
    decoding steps' tests (tests/parity_util.py); a pair in 8 bits is off by half a step more, at most 1 / 127 of its row's largest value."""
    from paper_2604_21215_amd import binding, torch_io as tio
    from tests.parity_util import TOL
    rng = np.random.default_rng(d + S)
    H, pos = d // 64, _lens(np.random.default_rng(S), S, most)
    pool = ref.Pool(rng, dtype, bits, S, H, pos, page, room=1)
    w, g = _layer(31, dtype, d, F)
    x = _rows(rng, dtype, S, d)
    ctx = _context(d, S, dtype, F=F, attn_scale=0.125, alibi_max_bias=alibi, resid_scale=0.7,
                   flags=binding.RT_FLAG_NORM_FREE if norm_free else 0)
    try:
        dl = tio.DeviceLayer(w, g, dtype)
        xd = tio.to_device(x, dtype)
        y = torch.full((S, d), 7.0, dtype=xd.dtype, device="cuda:0")
        before = pool.bits_of()
        ctx.rt_decode_step_paged(dl.struct, pool.cache(), xd, _ints(pos), most, y)
        assert ctx.engine_name() == "decode-paged" and ctx.engine_form() == "launches"
        ko, vo = (torch.full((S, 1, H, 64), 7.0, dtype=xd.dtype, device="cuda:0") for _ in range(2))
        ctx.rt_cache_read(pool.cache(), _ints(pos), None, ko, vo)
        torch.cuda.synchronize()
        after = pool.bits_of()
    finally:
        ctx.rt_destroy()
    w64, g64 = ({n: t.astype(np.float64) for n, t in m.items()} for m in (w, g))
    yr, kr, vr = ref.layer_step(w64, g64, x.astype(np.float64), [(pool.K[s], pool.V[s]) for s in range(S)], H, 0.125, alibi, 0.7,
                                norm_free=norm_free)
    got, gk, gv = _host(y), _host(ko)[:, 0], _host(vo)[:, 0]
    tab, touched = pool.table.cpu().numpy(), np.zeros(after[0].shape[:3], dtype=bool)
    norm = lambda a: np.linalg.norm(a.reshape(-1))  # noqa: E731
    for s in range(S):
        if pos[s] < 0:
            assert np.all(got[s] == 7) and np.all(gk[s] == 7) and np.all(gv[s] == 7)
            continue
        touched[tab[s, pos[s] // page], :, pos[s] % page] = True
        assert norm(got[s] - yr[s]) <= TOL[dtype] * norm(yr[s]), s
        branch = yr[s] - x[s].astype(np.float64)
        assert norm(got[s] - yr[s]) <= TOL[dtype] * norm(branch) + HALF[dtype] * norm(yr[s]), s
        for a, r in ((gk[s], kr[s]), (gv[s], vr[s])):
            coarse = np.sqrt(64 * ((np.abs(r).max(-1) / 127) ** 2).sum()) if bits else 0.0
            assert norm(a - r) <= TOL[dtype] * norm(r) + coarse, s
    for a, b in zip(after, before):   # one row of each sequence, and nothing else
        np.testing.assert_array_equal(a[~touched], b[~touched])


@pytest.mark.parametrize("dtype,d,S", [("bf16", 256, 3), ("bf16", 256, 20), ("f32", 192, 11), ("bf16", 512, 40)])
def test_step_on_the_plain_alus_agrees(dtype, d, S):
    """RT_FLAG_NO_MFMA: the same step on other kernels.  Both are within the tolerance of the float64 layer, so within twice of each other; the
    cached pairs of bf16 differ by a rounding where the sums fall on either side."""
    from paper_2604_21215_amd import binding, torch_io as tio
    from tests.parity_util import TOL
    H, pos = d // 64, _lens(np.random.default_rng(S), S, 100)
    w, g = _layer(12, dtype, d, 4 * d)
    dl = tio.DeviceLayer(w, g, dtype)
    x = tio.to_device(_rows(np.random.default_rng(1), dtype, S, d), dtype)
    got = []
    for flags in (0, binding.RT_FLAG_NO_MFMA):
        pool = ref.Pool(np.random.default_rng(d), dtype, 0, S, H, pos, 16, room=1)
        ctx = _context(d, S, dtype, attn_scale=0.125, flags=flags)
        try:
            y = torch.zeros_like(x)
            ctx.rt_decode_step_paged(dl.struct, pool.cache(), x, _ints(pos), 100, y)
            ko, vo = (torch.zeros((S, 1, H, 64), dtype=x.dtype, device="cuda:0") for _ in range(2))
            ctx.rt_cache_read(pool.cache(), _ints(pos), None, ko, vo)
            torch.cuda.synchronize()
            got.append([_host(t) for t in (y, ko, vo)])
        finally:
            ctx.rt_destroy()
    for a, b in zip(*got):
        assert np.linalg.norm(a - b) <= 2 * TOL[dtype] * np.linalg.norm(b) and np.linalg.norm(b) > 0


def test_step_beyond_its_bound_and_without_a_page():
    """pos > max_pos: y is NaN and nothing is cached; a wrong page for the new row: y as ever, nothing cached."""
    from paper_2604_21215_amd import torch_io as tio
    rng = np.random.default_rng(2)
    pos = [20, 32, 10]
    pool = ref.Pool(rng, "bf16", 0, 3, 4, pos, 16, room=1)
    w, g = _layer(8, "bf16", 256, 1024)
    dl = tio.DeviceLayer(w, g, "bf16")
    x = torch.randn((3, 256), device="cuda:0").bfloat16()
    ctx = _context(256, 3, "bf16", attn_scale=0.125)
    try:
        fine = torch.zeros_like(x)
        keep = pool.Kd.clone(), pool.Vd.clone()
        ctx.rt_decode_step_paged(dl.struct, pool.cache(), x, _ints(pos), 32, fine)
        torch.cuda.synchronize()
        pool.Kd.copy_(keep[0]); pool.Vd.copy_(keep[1])
        pool.table[1, 2] = -1
        before = pool.bits_of()
        y = torch.zeros_like(x)
        ctx.rt_decode_step_paged(dl.struct, pool.cache(), x, _ints([20, 32, 33]), 32, y)
        torch.cuda.synchronize()
        assert torch.equal(y[:2], fine[:2]) and bool(torch.isnan(y[2]).all())
        tab = pool.table.cpu().numpy()
        for a, b in zip(before, pool.bits_of()):
            diff = np.argwhere((a != b).reshape(a.shape[0], 4, 16, -1).any(-1))
            assert {(p, r) for p, _, r in diff.tolist()} == {(int(tab[0, 1]), 4)}
    finally:
        ctx.rt_destroy()


def test_captured_step_reads_its_positions_at_every_replay():
    """A step, the attention by itself and the read of the new pairs in one graph; positions, inputs and the page table change between the
    replays, which run among eager work of the same context.  Every replay equals the eager calls on the same state, bit for bit."""
    from paper_2604_21215_amd import binding, torch_io as tio
    rng = np.random.default_rng(4)
    S, d, H, most = 5, 256, 4, 540
    for bits in (0, 8):
        pool = ref.Pool(rng, "bf16", bits, S, H, [500, 300, 40, 500, 64], 16, room=3)
        w, g = _layer(9, "bf16", d, 4 * d)
        dl = tio.DeviceLayer(w, g, "bf16")
        st = torch.cuda.Stream()
        ctx = _context(d, S, "bf16", attn_scale=0.125, alibi_max_bias=8.0, stream=st.cuda_stream, reserve=binding.RT_RESERVE_PAGED)
        try:
            x, y = torch.zeros((S, d), device="cuda:0").bfloat16(), torch.zeros((S, d), device="cuda:0").bfloat16()
            q, out = torch.zeros((S, H, 64), device="cuda:0").bfloat16(), torch.zeros((S, H, 64), device="cuda:0").bfloat16()
            lse = torch.zeros((S, H), device="cuda:0")
            ko, vo = (torch.zeros((S, 1, H, 64), device="cuda:0").bfloat16() for _ in range(2))
            pos = _ints([0] * S)
            def calls():
                ctx.rt_decode_step_paged(dl.struct, pool.cache(), x, pos, most, y)
                ctx.rt_cache_read(pool.cache(), pos, None, ko, vo)
                ctx.rt_paged_attention(pool.cache(), pos, most, q, None, None, out, lse)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                calls()
            for rep, at in enumerate(([500, 300, 40, -1, 64], [501, 301, -1, 17, 65], [13, 299, 41, 500, 1], [0, 0, 0, 0, 0])):
                gen_ = torch.Generator(device="cuda:0")
                gen_.manual_seed(rep)
                x.copy_(torch.randn((S, d), generator=gen_, device="cuda:0")); q.copy_(torch.randn((S, H, 64), generator=gen_, device="cuda:0"))
                pos.copy_(torch.tensor(at, dtype=torch.int32))
                start = [t.clone() for t in (pool.Kd, pool.Vd, pool.K_exp, pool.V_exp) if t is not None]
                got = []
                for eager in (True, False):
                    for t, s0 in zip((t for t in (pool.Kd, pool.Vd, pool.K_exp, pool.V_exp) if t is not None), start):
                        t.copy_(s0)
                    for t in (y, out, lse, ko, vo):
                        t.zero_()
                    torch.cuda.synchronize()
                    with torch.cuda.stream(st):
                        calls() if eager else graph.replay()
                    torch.cuda.synchronize()
                    got.append([t.clone() for t in (y, out, lse, ko, vo)])
                for a, b in zip(*got):
                    assert torch.equal(a, b), rep
                assert float(got[0][0].float().abs().max()) > 0
        finally:
            ctx.rt_destroy()


def test_capture_without_scratch_is_refused():
    """A capture cannot allocate: the call says so, and the context works afterwards."""
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(4)
    pool = ref.Pool(rng, "bf16", 0, 1, 2, [20], 16)
    st = torch.cuda.Stream()
    ctx = _context(128, 1, "bf16", stream=st.cuda_stream)
    q, out, n = torch.randn((1, 2, 64), device="cuda:0").bfloat16(), torch.zeros((1, 2, 64), device="cuda:0").bfloat16(), _ints([20])
    torch.cuda.synchronize()
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out.zero_()
            with pytest.raises(binding.RTError, match="RT_ERR_STATE"):
                ctx.rt_paged_attention(pool.cache(), n, 20, q, None, None, out)
        with torch.cuda.stream(st):
            ctx.rt_paged_attention(pool.cache(), n, 20, q, None, None, out)
        torch.cuda.synchronize()
        assert float(out.float().abs().max()) > 0
        assert ctx.workspace_bytes() > 16 << 20
    finally:
        ctx.rt_destroy()


def test_shared_prefix_pages():
    """Two sequences whose first pages are the same ones."""
    rng = np.random.default_rng(6)
    pool = ref.Pool(rng, "bf16", 0, 2, 2, [100, 90], 16)
    pool.table[1, :3] = pool.table[0, :3].clone()
    q = torch.randn((2, 2, 64), device="cuda:0").bfloat16()
    ctx = _context(128, 2, "bf16", attn_scale=0.125)
    try:
        out = torch.zeros_like(q)
        ctx.rt_paged_attention(pool.cache(), _ints([100, 90]), 100, q, None, None, out)
        torch.cuda.synchronize()
    finally:
        ctx.rt_destroy()
    K = [pool.K[0], np.concatenate((pool.K[0][:48], pool.K[1][48:]))]
    V = [pool.V[0], np.concatenate((pool.V[0][:48], pool.V[1][48:]))]
    for s in range(2):
        o, _, bound, _ = ref.attention(_host(q)[s], K[s], V[s], None, None, 0.125, 0.0, HALF["bf16"])
        assert np.all(np.abs(_host(out)[s] - o) <= bound)


def test_refusals_leave_outputs_and_context_alone():
    """The checks of paged_args_check.cpp reach the entry points: status, reason, nothing enqueued."""
    from paper_2604_21215_amd import binding
    rng = np.random.default_rng(7)
    pool = ref.Pool(rng, "bf16", 8, 2, 2, [20, 20], 16)
    ctx = _context(128, 2, "bf16")
    q = torch.randn((3, 2, 64), device="cuda:0").bfloat16()
    out, n = torch.full_like(q, 7.0), _ints([20, 20, 20])
    k = torch.zeros((2, 1, 2, 64), device="cuda:0").bfloat16()
    w = binding.rt_layer_weights(*([1 << 30] * 6))
    try:
        before = pool.bits_of()
        cache = pool.cache()
        wrong = pool.cache()
        wrong.page_len = 24
        four = pool.cache()
        four.bits = 4
        for call, status, text in ((lambda: ctx.rt_paged_attention(cache, n, 20, q, None, None, out), "INVALID_ARG", "max_batch"),
                                   (lambda: ctx.rt_paged_attention(cache, n, 1000, q[:2], None, None, out[:2]), "INVALID_ARG", "max_len"),
                                   (lambda: ctx.rt_paged_attention(cache, n, 20, q[:2], None, None, q[:2]), "INVALID_ARG", "overlap"),
                                   (lambda: ctx.rt_paged_attention(wrong, n, 20, q[:2], None, None, out[:2]), "INVALID_ARG", "page_len"),
                                   (lambda: ctx.rt_paged_attention(four, n, 20, q[:2], None, None, out[:2]), "UNSUPPORTED", "8 bits"),
                                   (lambda: ctx.rt_cache_write(wrong, n, None, k, k), "INVALID_ARG", "page_len"),
                                   (lambda: ctx.rt_cache_read(cache, n, None, k, k), "INVALID_ARG", "overlap"),
                                   (lambda: ctx.rt_decode_step_paged(w, cache, q[:2], n, 1000, out[:2]), "INVALID_ARG", "max_pos"),
                                   (lambda: ctx.rt_decode_step_paged(binding.rt_layer_weights(), cache, q[:2], n, 20, out[:2]), "INVALID_ARG", "weight")):
            with pytest.raises(binding.RTError, match=status) as e:
                call()
            assert text in str(e.value)
        torch.cuda.synchronize()
        assert bool((out == 7).all())
        for a, b in zip(before, pool.bits_of()):
            np.testing.assert_array_equal(a, b)
        ctx.rt_paged_attention(cache, n, 20, q[:2], None, None, out[:2])   # still usable
        torch.cuda.synchronize()
        assert not bool((out[:2] == 7).any())
    finally:
        ctx.rt_destroy()
