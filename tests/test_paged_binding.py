"""What the binding refuses before the library follows an address, on the CPU: a context that never calls the library."""
import pytest

torch = pytest.importorskip("torch")

from paper_2604_21215_amd import binding  # noqa: E402

H, S, ENTRIES = 2, 3, 4
D = 64 * H
CPU = -1   # what a tensor on the host calls its device


def _ctx(dtype=binding.RT_BF16, max_batch=8, device=CPU):
    ctx = binding.RTContext.__new__(binding.RTContext)
    ctx.cfg = binding.rt_config(D, H, 64, 256, max_batch, 1, dtype, 0, 1.0, 1.0, 1e-6, 0, device)
    ctx.calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: ctx.calls.append((name, a)) or 0

    ctx._L, ctx._ctx = Library(), None
    return ctx


def _i32(n, fill=0):
    return torch.full((n,), fill, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _cache(heads=H, dtype=torch.bfloat16, lines=S, bits=0):
    shape = (5, heads, 16, 64)
    exps = [torch.zeros(shape[:3], dtype=torch.uint8) if bits else None for _ in range(2)]
    return binding.make_cache(*(torch.zeros(shape, dtype=torch.int8 if bits else dtype) for _ in range(2)),
                              torch.zeros((lines, ENTRIES), dtype=torch.int32), *exps)


def _refused(ctx, call, text=""):
    before = len(ctx.calls)
    with pytest.raises(binding.RTError, match="RT_ERR_INVALID_ARG") as e:
        call()
    assert len(ctx.calls) == before and text in str(e.value)


@pytest.mark.parametrize("bits", [0, 8])
def test_a_cache_fits_its_context(bits):
    """More sequences than lines of the table, another number of heads, rows of another type, another device."""
    ctx = _ctx()
    kv, out, q = _bf16(S, 1, H, 64), _bf16(S, H, 64), _bf16(S, H, 64)
    calls = (lambda c, n=S, ctx=ctx: ctx.rt_cache_write(c, _i32(n), None, kv[:1].expand(n, 1, H, 64).contiguous(), kv[:1].expand(n, 1, H, 64).contiguous()),
             lambda c, n=S, ctx=ctx: ctx.rt_cache_read(c, _i32(n), _i32(n), _bf16(n, 1, H, 64), _bf16(n, 1, H, 64)),
             lambda c, n=S, ctx=ctx: ctx.rt_paged_attention(c, _i32(n), 20, _bf16(n, H, 64), None, None, _bf16(n, H, 64)),
             lambda c, n=S, ctx=ctx: ctx.rt_decode_step_paged(binding.rt_layer_weights(), c, _bf16(n, D), _i32(n), 20, _bf16(n, D)))
    wrong = [_cache(heads=H + 1, bits=bits), _cache(heads=1, bits=bits)] + ([] if bits else [_cache(dtype=torch.float32)])
    for call in calls:
        call(_cache(bits=bits))
        call(_cache(bits=bits, lines=S + 2))
        assert len(ctx.calls) == 2
        del ctx.calls[:]
        for c in wrong:
            _refused(ctx, lambda: call(c), "heads")
        _refused(ctx, lambda: call(_cache(bits=bits), S + 1), "lines")
        other = _ctx(device=0)
        _refused(other, lambda: call(_cache(bits=bits), ctx=other), "device")
    assert out.shape == q.shape


def test_make_cache_refuses():
    K, V, table = _bf16(5, H, 16, 64), _bf16(5, H, 16, 64), torch.zeros((S, ENTRIES), dtype=torch.int32)
    K8, exp = K.to(torch.int8), torch.zeros((5, H, 16), dtype=torch.uint8)
    c = binding.make_cache(K, V, table)
    assert (c.pages, c.page_len, c.bits, c.table_stride) == (5, 16, 0, ENTRIES)
    c = binding.make_cache(K8, K8.clone(), torch.zeros((S + 1, 9), dtype=torch.int32)[:S], exp, exp.clone())
    assert (c.pages, c.page_len, c.bits, c.table_stride) == (5, 16, 8, 9)
    for args in ((K.half(), V.half(), table), (K.to(torch.int16), V.to(torch.int16), table), (K.to(torch.int32), V.to(torch.int32), table), (K, V, table.float()), (K, V, table.long()), (K, V, torch.zeros((ENTRIES, S), dtype=torch.int32).t()),
                 # columns of a wider table: its other columns would be followed, and read past the end behind the last line
                 (K, V, torch.zeros((S, 9), dtype=torch.int32)[:, :ENTRIES]), (K, V, torch.zeros((S, 9), dtype=torch.int32)[:, 5:]),
                 (K, V[:4], table), (K, V.float(), table), (K.transpose(1, 2), V.transpose(1, 2), table), (K[..., :32], V[..., :32], table),
                 (K[..., :32].contiguous(), V[..., :32].contiguous(), table), (K8, K8, table), (K, V, table, exp, exp), (K8, K8, table, exp, None),
                 (K8, K8, table, None, exp), (K8, K8, table, exp, exp[:4]), (K8, K8, table, exp.int(), exp.int()), (K[0], V[0], table)):
        with pytest.raises(binding.RTError, match="RT_ERR_INVALID_ARG"):
            binding.make_cache(*args)


def _wrong_ints(n):
    return (_i32(n).long(), _i32(n).float(), _i32(n - 1), _i32(2 * n)[::2], _i32(n).to(torch.int16))


def test_attention_refuses():
    ctx, c = _ctx(), _cache()
    q, kt, vt, out, lse, lens = _bf16(S, H, 64), _bf16(S, H, 64), _bf16(S, H, 64), _bf16(S, H, 64), torch.zeros((S, H)), _i32(S)
    go = lambda **k: ctx.rt_paged_attention(c, *({**dict(lens=lens, most=20, q=q, kt=kt, vt=vt, out=out, lse=lse), **k}.values()))  # noqa: E731
    qkv = _bf16(S, 3 * D + 64)
    for good in (dict(), dict(kt=None, vt=None, lse=None), dict(q=q.view(S, D), out=out.view(S, D)), dict(lens=_i32(S + 1), out=_bf16(S + 1, H, 64)),
                 dict(q=qkv[:, :D], kt=qkv[:, D:2 * D], vt=qkv[:, 2 * D:3 * D]), dict(q=qkv[:, :D].unflatten(1, (H, 64))), dict(lse=torch.zeros((S + 1, H)))):
        go(**good)
    strides = [(a[6], a[9], a[11]) for _, a in ctx.calls]
    W = 3 * D + 64
    assert strides == [(D, D, D), (D, D, D), (D, D, D), (D, D, D), (W, W, D), (W, D, D), (D, D, D)]
    one = _ctx()
    one.rt_paged_attention(c, _i32(1), 20, qkv[:1, :D], qkv[:1, D:2 * D], qkv[:1, 2 * D:3 * D], out[:1], None)   # one row has no stride
    assert [(a[6], a[9], a[11]) for _, a in one.calls] == [(D, D, D)]
    rows = (_bf16(S, 64, H).transpose(1, 2), _bf16(S, H, 128)[..., ::2], _bf16(D, S).t(), q.float(), q.half(), _bf16(S - 1, H, 64), _bf16(S, H + 1, 64),
            _bf16(S, D + 1)[:, :D - 1], _bf16(S, 2 * D)[:, ::2], _bf16(S, H, 65)[..., :64])
    for w in rows:
        for name in ("kt", "vt", "out"):
            _refused(ctx, lambda: go(**{name: w}))
        if w.shape[0] == S:
            _refused(ctx, lambda: go(q=w))
    _refused(ctx, lambda: go(vt=qkv[:, 2 * D:3 * D]), "stride")
    for w in _wrong_ints(S):
        _refused(ctx, lambda: go(lens=w), "int32")
    for w in (lse.bfloat16(), lse[:2], torch.zeros((H, S)).t(), lse.to(torch.int32), lse.double()):
        _refused(ctx, lambda: go(lse=w), "lse")


def test_rows_of_pairs_refuse():
    ctx, c = _ctx(), _cache()
    k, v = _bf16(S, 5, H, 64), _bf16(S, 5, H, 64)
    for name in ("rt_cache_write", "rt_cache_read"):
        f = getattr(ctx, name)
        f(c, _i32(S), None, k, v)
        f(c, _i32(S + 1), _i32(S), _bf16(5, S, H, 64).transpose(0, 1), _bf16(5, S, H, 64).transpose(0, 1))
        f(c, _i32(S), None, *_bf16(S, 5, 2, H, 64).unbind(2))
        f(c, _i32(1), None, _bf16(5, 1, H, 64).transpose(0, 1), _bf16(1, 5, H, 64))
        assert [(n, a[8:]) for n, a in ctx.calls] == [(name, (5 * D, D)), (name, (D, S * D)), (name, (10 * D, 2 * D)), (name, (0, D))]
        del ctx.calls[:]
        for w in _wrong_ints(S):
            _refused(ctx, lambda: f(c, w, None, k, v), "int32")
            _refused(ctx, lambda: f(c, _i32(S), w, k, v), "int32")
        for a, b in ((k.float(), v.float()), (k, v.float()), (k.float(), v), (k.half(), v.half()), (k, v[:, :4]), (k, v.transpose(0, 1)), (k[0], v[0]),
                     (_bf16(S, 5, 64, H).transpose(2, 3), _bf16(S, 5, 64, H).transpose(2, 3)), (_bf16(S, 5, H + 1, 64), _bf16(S, 5, H + 1, 64)),
                     (_bf16(S, 5, H, 32), _bf16(S, 5, H, 32)), (_bf16(S, 5, H, 128)[..., ::2], _bf16(S, 5, H, 128)[..., ::2])):
            _refused(ctx, lambda: f(c, _i32(S), None, a, b))


def test_step_refuses():
    ctx, c, w = _ctx(), _cache(), binding.rt_layer_weights()
    x, y, pos = _bf16(S, D), _bf16(S, D), _i32(S)
    ctx.rt_decode_step_paged(w, c, x, pos, 20, y)
    ctx.rt_decode_step_paged(w, c, x.view(S, H, 64), _i32(S + 2), 20, _bf16(S + 1, D))
    assert len(ctx.calls) == 2
    for bad in (_bf16(D, S).t(), _bf16(S, 2 * D)[:, :D], _bf16(S, D - 1), x.float(), _bf16(S - 1, D)):
        if bad.shape[0] == S:
            _refused(ctx, lambda: ctx.rt_decode_step_paged(w, c, bad, pos, 20, y))
        _refused(ctx, lambda: ctx.rt_decode_step_paged(w, c, x, pos, 20, bad))
    for bad in _wrong_ints(S):
        _refused(ctx, lambda: ctx.rt_decode_step_paged(w, c, x, bad, 20, y), "int32")


def test_read_out_refuses():
    ctx, vocab = _ctx(), 10
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    base = dict(codes=u8(vocab, D // 2), exps=u8(vocab, D // 32), g=_bf16(D), z=_bf16(S, D), stride=D, B=S, logits=torch.zeros((S, vocab)))
    go = lambda **k: ctx.rt_lm_head_mx4(*{**base, **k}.values())  # noqa: E731
    good = (dict(), dict(g=None), dict(z=_bf16(S, 1, D)), dict(z=_bf16(S, 3, D)[:, 1], stride=3 * D), dict(z=_bf16(1, 7, D)[:, 6], stride=7 * D, B=1),
            dict(z=_bf16(S, 2 * D), stride=2 * D), dict(logits=torch.zeros((S + 1, vocab))))
    for k in good:
        go(**k)
    assert len(ctx.calls) == len(good)
    for k in (dict(codes=u8(vocab, D)), dict(codes=u8(vocab, D)[:, ::2]), dict(codes=torch.zeros((vocab, D // 2), dtype=torch.int32)), dict(exps=u8(vocab - 1, D // 32)), dict(exps=torch.zeros((vocab, D // 32), dtype=torch.int32)),
              dict(exps=u8(D // 32, vocab).t()), dict(g=torch.zeros(D)), dict(g=_bf16(D - 1)), dict(g=_bf16(2 * D)[::2]), dict(z=torch.zeros((S, D))),
              dict(z=_bf16(S - 1, D)), dict(stride=2 * D), dict(z=_bf16(S, 2 * D)[:, :D]), dict(z=_bf16(D, S).t()), dict(logits=torch.zeros((S, vocab)).bfloat16()),
              dict(logits=torch.zeros((S, vocab - 1))), dict(logits=torch.zeros((vocab, S)).t())):
        _refused(ctx, lambda: go(**k))


def test_tensors_of_another_device_are_refused():
    """Every tensor of a call but one on the context's device (here the host)."""
    vocab, u8 = 10, lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    z, w = torch.zeros((S, H)), binding.rt_layer_weights()
    calls = (("rt_cache_write", lambda: [_i32(S), _i32(S), _bf16(S, 5, H, 64), _bf16(S, 5, H, 64)]),
             ("rt_cache_read", lambda: [_i32(S), _i32(S), _bf16(S, 5, H, 64), _bf16(S, 5, H, 64)]),
             ("rt_paged_attention", lambda: [_i32(S), 20, _bf16(S, H, 64), _bf16(S, H, 64), _bf16(S, H, 64), _bf16(S, H, 64), z]),
             ("rt_decode_step_paged", lambda: [_bf16(S, D), _i32(S), 20, _bf16(S, D)]),
             ("rt_lm_head_mx4", lambda: [u8(vocab, D // 2), u8(vocab, D // 32), _bf16(D), _bf16(S, D), D, S, torch.zeros((S, vocab))]))

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1

    for name, args in calls:
        ctx, c = _ctx(), _cache()
        before = {"rt_lm_head_mx4": [], "rt_decode_step_paged": [w, c]}.get(name, [c])
        getattr(ctx, name)(*before, *args())
        assert len(ctx.calls) == 1
        for i, a in enumerate(args()):
            if torch.is_tensor(a):
                moved = args()
                moved[i] = a.as_subclass(Elsewhere)
                _refused(ctx, lambda: getattr(ctx, name)(*before, *moved), "device")
