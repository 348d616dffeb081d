"""A stack served from pages: prompts of different lengths prefilled together, their pairs moved into pages (storage dtype and 8 bits),
tokens generated at every sequence's own position, a sequence that ends and another that takes its place and its pages, and the read-out
with 4-bit weights.  Against the CPU oracle: the output of a layer at a position depends on earlier positions only, so every generated
token's rows are those of the oracle's prefill of the whole sequence."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests.parity_util import TOL, rel_err_rows
from tests.test_paged_args import mx4_values

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

L, B, VOCAB, STEPS = 3, 4, 500, 6


def _stack(oracle, dtype, d):
    from paper_2604_21215_amd import binding, torch_io as tio
    from paper_2604_21215_amd.stack import DeviceStack
    H, F = d // 64, 4 * d
    rnd = gen.round_to_bf16 if dtype == "bf16" else (lambda a: a)
    emb, head = rnd(gen.normal(5, 3, (VOCAB, d), 1.0)), rnd(gen.normal(5, 4, (VOCAB, d), 0.02))
    g_final = rnd((1 + 0.1 * gen.normal(5, 6, (d,))).astype(np.float32))
    ctx = binding.RTContext(d, H, F, B, 128, dtype, resid_scale=L ** -0.5, rms_eps=1e-6, attn_scale=0.125, alibi_max_bias=8.0,
                            stream=torch.cuda.current_stream().cuda_stream, reserve=binding.RT_RESERVE_PAGED)
    ws = [gen.make_layer_weights(77, l, d, F, dtype) for l in range(L)]
    ds = DeviceStack(ctx, [tio.DeviceLayer(w, None, dtype) for w in ws], emb, head, g_final, dtype)
    os_ = oracle.Stack([oracle.Layer({k: v.astype(np.float64) for k, v in w.items()}, H, alpha=L ** -0.5, eps=1e-6, attn_scale=0.125,
                                     alibi_max_bias=8.0) for w in ws], emb.astype(np.float64), head.astype(np.float64),
                       g_final.astype(np.float64), eps=1e-6)
    return ctx, ds, os_


@pytest.mark.parametrize("dtype,d,bits", [("f32", 128, 0), ("bf16", 256, 0), ("bf16", 256, 8), ("f32", 128, 8)])
def test_generation_from_pages(oracle, dtype, d, bits):
    from paper_2604_21215_amd.paged import PagedCaches
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    rng = np.random.default_rng(d + bits)
    ids = rng.integers(0, VOCAB, (2 * B, 100)).astype(np.int32)
    ctx, ds, os_ = _stack(oracle, dtype, d)
    # 8 bits: a row's step is at most a 63rd of its largest value, some 0.05 of its root mean square, so a key or a value is off by
    # 0.015 of its norm; logits 0.125 <q, k> with |q| = |k| = 8 by 0.015, their weights and the values they add up by 0.02 at most; three layers
    tol = TOL[dtype] + (0.02 * np.sqrt(3) if bits else 0.0)
    ref = []
    for half in (ids[:B], ids[B:]):
        layers, _ = os_.prefill(half, 100, 100)
        ref.append([y for y, _, _ in layers])
    caches = PagedCaches(L, d // 64, B, 96, 14, page_len=16, bits=bits, dtype=dtype)
    try:
        lens = np.array([40, 17, 1, 30])
        ds.prefill(torch.from_numpy(ids[:B]).to("cuda:0"), 40, 40)
        ds.into_pages(caches, lens)
        whose = [(0, b) for b in range(B)]
        pos = lens.copy()

        def generate(n):
            for _ in range(n):
                caches.reserve([p + 1 if p >= 0 else 0 for p in pos])
                tok = [ids[B * whose[s][0] + whose[s][1], pos[s]] if pos[s] >= 0 else -7 for s in range(B)]
                logits, rows = ds.decode_step_paged(caches, torch.tensor(tok, dtype=torch.int32, device="cuda:0"),
                                                    torch.tensor(pos, dtype=torch.int32, device="cuda:0"), 95)
                torch.cuda.synchronize()
                got, lg = rows.float().cpu().numpy().astype(np.float64), logits.cpu().numpy().astype(np.float64)
                for s in range(B):
                    if pos[s] < 0:
                        assert np.all(got[:, s] == 0)
                        continue
                    half, b = whose[s]
                    for l in range(L):
                        want = ref[half][l][b, pos[s]]
                        assert rel_err_rows(got[l, s], want) <= tol, (s, l, pos[s])
                    want = oracle.lm_head(os_.W_lm, got[L - 1, s][None], os_.g_final, eps=1e-6)[0]
                    assert rel_err_rows(lg[s], want) <= 1e-5, s
                    pos[s] += 1

        generate(STEPS)
        pages_before = len(caches.free)
        caches.release(1)
        assert len(caches.free) == pages_before + 2
        pos[1] = -1
        generate(2)
        # another sequence takes place 1: prefilled with others, whose rows are not wanted
        ds.prefill(torch.from_numpy(ids[B:]).to("cuda:0"), 33, 33)
        ds.into_pages(caches, [-1, 33, -1, -1])
        whose[1], pos[1] = (1, 1), 33
        generate(STEPS)
        with pytest.raises(MemoryError):
            caches.reserve([96, 96, 96, 96])
        with pytest.raises(ValueError):
            caches.reserve([97, 0, 0, 0])
        # the 4-bit read-out of the same rows
        ds.pack_lm_head()
        one = torch.tensor(pos, dtype=torch.int32, device="cuda:0")
        caches.reserve(pos + 1)
        logits, rows = ds.decode_step_paged(caches, torch.tensor([3, 5, 7, 9], dtype=torch.int32, device="cuda:0"), one, 95, head4=True)
        torch.cuda.synchronize()
        z = rows[L - 1].float().cpu().numpy().astype(np.float64)
        n = z / np.sqrt((z * z).mean(-1, keepdims=True) + 1e-6) * os_.g_final
        W4 = mx4_values(*(t.cpu().numpy() for t in ds.head4))
        assert np.linalg.norm(logits.cpu().numpy() - n @ W4.T) <= 1e-6 * np.linalg.norm(n @ W4.T)
        # and packed weights stand for the matrix: each is off by at most a third of itself or half of the smallest step (0.25 / 6 of
        # the largest at most), at random: 0.3 of the norm is far above, unrelated weights would be off by 1.4
        exact = n @ os_.W_lm.T
        assert np.linalg.norm(n @ W4.T - exact) <= 0.3 * np.linalg.norm(exact)
    finally:
        ctx.rt_destroy()
