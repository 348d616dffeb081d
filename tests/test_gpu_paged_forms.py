"""Decoding steps from pages on every form of the kernels (tests/paged_forms.py; which call takes which form: tests/test_paged_plans.py),
held to float64 closely enough that a rounding of any vector on the way shows.  And an attention of sixteen wavefronts in several parts."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests import paged_forms as forms
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")


def _ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("form", forms.FORMS, ids=forms.NAMES)
def test_step(form):
    from paper_2604_21215_amd import binding, torch_io as tio
    name, dtype, bits, d, F, most, page, alibi, scale, pos = form[:10]
    S, H = len(pos), d // 64
    rng = np.random.default_rng(d + S + most)
    x, w, g = forms.inputs(form)
    pool = ref.Pool(rng, dtype, bits, S, H, pos, page, room=1)
    ctx = binding.RTContext(d, H, F, S, 1, dtype, rms_eps=1e-6, attn_scale=scale, alibi_max_bias=alibi, resid_scale=0.75,
                            stream=torch.cuda.current_stream().cuda_stream)
    try:
        dl, xd = tio.DeviceLayer(w, g, dtype), tio.to_device(x, dtype)
        outs = []
        before = pool.bits_of()
        for _ in range(2):
            y = torch.full((S, d), 7.0, dtype=xd.dtype, device="cuda:0")
            ko, vo = (torch.full((S, 1, H, 64), 7.0, dtype=xd.dtype, device="cuda:0") for _ in range(2))
            ctx.rt_decode_step_paged(dl.struct, pool.cache(), xd, _ints(pos), most, y)
            ctx.rt_cache_read(pool.cache(), _ints(p if p <= most else -1 for p in pos), None, ko, vo)
            torch.cuda.synchronize()
            outs.append([tio.to_host(t) for t in (y, ko, vo)])
        after = pool.bits_of()
    finally:
        ctx.rt_destroy()
    for a, b in zip(*outs):
        np.testing.assert_array_equal(a, b)
    y, k, v = outs[0][0], outs[0][1][:, 0], outs[0][2][:, 0]
    live = np.array([0 <= p <= most for p in pos])
    for s in np.flatnonzero(~live):
        assert np.all(y[s] == 7) if pos[s] < 0 else np.all(np.isnan(y[s]))
        assert np.all(k[s] == 7) and np.all(v[s] == 7)
    tab, touched = pool.table.cpu().numpy(), np.zeros(after[0].shape[:3], dtype=bool)
    for s in np.flatnonzero(live):
        touched[tab[s, pos[s] // page], :, pos[s] % page] = True
    for a, b in zip(after, before):   # one row of each live sequence, and nothing else
        np.testing.assert_array_equal(a[~touched], b[~touched])
    f64 = lambda m: {n: t.astype(np.float64) for n, t in m.items()}  # noqa: E731
    want = forms.step(f64(w), f64(g), x[live].astype(np.float64), [(pool.K[s], pool.V[s]) for s in np.flatnonzero(live)], H, scale, alibi, 0.75)
    for what, got, u in zip("ykv", (y[live], k[live], v[live]), want):
        if what != "y" and bits:
            top = np.abs(u).max(-1, keepdims=True) * np.array([1 - 2.0 ** -11, 1 + 2.0 ** -11])
            same = ref.quantise(top[..., None])[1]           # a largest value next to the end of a step may take the next one
            rows = same[..., 0] == same[..., 1]
            assert rows.mean() > 0.9
            flips, allowed = forms.moved(got[rows], u[rows], forms.row_step(u[rows]))
        elif dtype == "bf16":
            flips, allowed = forms.moved(got, u, forms.bf16_ulp(u))
        else:
            # fp32: 2^-24 for each of up to 640 terms in eight running sums and their joins, 2^-20 of a product at random, times the logits' 8 sqrt(2)
            err = np.linalg.norm(got - u, axis=-1) / np.linalg.norm(u, axis=-1)
            assert np.all(err <= 2.0 ** -16), (name, what, err.max())
            continue
        print(name, what, "moved", flips, "of", u.size, "allowed", int(allowed))
        assert flips <= allowed, (name, what, flips, allowed)
        # and each by its rounding (half of the spacing, which may double at the next power of two) and its error, DELTA of the row's root mean
        # square or eight times that for the largest of 266112: an element of 2^-20 of its row has a spacing of 2^-28, far below its error of
        # up to 2^-15, so that places are no measure for each element
        space, rows = (forms.row_step(u), rows) if what != "y" and bits else (forms.bf16_ulp(u), slice(None))
        assert np.all((np.abs(got - u) <= space + 8 * forms.DELTA * np.sqrt((u ** 2).mean(-1, keepdims=True)))[rows]), (name, what)


def test_attention_of_sixteen_wavefronts_in_parts():
    from paper_2604_21215_amd import binding, torch_io as tio
    S, H, most = 17, 16, 16384
    rng = np.random.default_rng(2)
    lens = forms._few(S, 16384, 0, -1, 8193, 8192, 12000)
    pool = ref.Pool(rng, "bf16", 0, S, H, lens, 128)
    q = gen.round_to_bf16(rng.standard_normal((S, H, 64)).astype(np.float32))
    pair = [gen.round_to_bf16(rng.standard_normal((S, H, 64)).astype(np.float32)) for _ in range(2)]
    ctx = binding.RTContext(64 * H, H, 64, S, 1, "bf16", rms_eps=1e-6, attn_scale=0.125, stream=torch.cuda.current_stream().cuda_stream)
    try:
        qd, kd, vd = (tio.to_device(t, "bf16") for t in [q] + pair)
        out, lse = torch.full_like(qd, 7.0), torch.full((S, H), 7.0, device="cuda:0")
        ctx.rt_paged_attention(pool.cache(), _ints(lens), most, qd, kd, vd, out, lse)
        torch.cuda.synchronize()
        got, got_lse = tio.to_host(out), tio.to_host(lse)
    finally:
        ctx.rt_destroy()
    x = [t.astype(np.float64) for t in [q] + pair]
    for s in range(S):
        if lens[s] < 0:
            assert np.all(got[s] == 7) and np.all(got_lse[s] == 7)
            continue
        o, l, bound, lbound = ref.attention(x[0][s], pool.K[s], pool.V[s], x[1][s], x[2][s], 0.125, 0.0, HALF["bf16"])
        assert np.all(np.abs(got[s] - o) <= bound) and np.all(np.abs(got_lse[s] - l) <= lbound), s
