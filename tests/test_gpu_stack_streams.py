"""A stack whose context has a stream of its own, called while torch's current stream is another: what a call fills, copies and drops is
ordered with the context's kernels, however late the other stream is."""
import numpy as np
import pytest

from tests.test_gpu_paged_stack import B, VOCAB, L, _stack

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture
def served(oracle):
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx, ds, _ = _stack(oracle, "bf16", 256)
    ids = torch.from_numpy(np.random.default_rng(3).integers(0, VOCAB, (B, 60)).astype(np.int32)).to("cuda:0")
    torch.cuda.synchronize()
    yield st, ds, ids
    torch.cuda.synchronize()
    ctx.rt_destroy()


def _busy(stream):
    """Some 30 ms of work."""
    with torch.cuda.stream(stream):
        a = torch.full((8192, 8192), 0.01, device="cuda:0").bfloat16()
        for _ in range(30):
            torch.mm(a, a)


def _caches(bits=0):
    from paper_2604_21215_amd.paged import PagedCaches
    return PagedCaches(L, 4, B, 96, 24, page_len=16, bits=bits, dtype="bf16")


@pytest.mark.parametrize("wavefront", [False, True])
def test_a_call_does_not_wait_for_and_is_not_spoilt_by_another_stream(served, wavefront):
    st, ds, ids = served
    pos, tokens = torch.tensor([40, 3, -1, 17], dtype=torch.int32, device="cuda:0"), ids[:, 40].contiguous()
    got = []
    for late in (False, True):
        caches = _caches()
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.default_stream() if late else st):
            if late:
                _busy(torch.cuda.current_stream())
            first = ds.prefill(ids, 40, 50, wavefront=wavefront)
            pairs = list(ds.K) + list(ds.V)
            logits0, rows0 = ds.decode_step(ids, 40)
        torch.cuda.synchronize()
        pairs = [t.clone() for t in pairs]
        with torch.cuda.stream(st):
            ds.into_pages(caches, [40, 3, -1, 17])
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.default_stream() if late else st):
            if late:
                _busy(torch.cuda.current_stream())
            logits, rows = ds.decode_step_paged(caches, tokens, pos, 95)
        torch.cuda.synchronize()
        assert float(rows[:, [0, 1, 3]].float().abs().amax(-1).min()) > 0 and float(rows[:, 2].float().abs().max()) == 0
        got.append([first, logits0, rows0, logits[[0, 1, 3]], rows] + pairs)
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_into_pages_keeps_its_numbers_until_they_are_read(served):
    """The context's stream is late; the memory of the lengths is not given to the next tensors meanwhile."""
    st, ds, ids = served
    with torch.cuda.stream(st):
        ds.prefill(ids, 40, 40)
    got = []
    for late in (False, True):
        caches = _caches(8)
        torch.cuda.synchronize()
        if late:
            _busy(st)
            ds.into_pages(caches, [40, 3, -1, 17])
            for _ in range(300):
                torch.full((B,), 77, dtype=torch.int32, device="cuda:0")
        else:
            with torch.cuda.stream(st):
                ds.into_pages(caches, [40, 3, -1, 17])
        torch.cuda.synchronize()
        got.append(caches.K + caches.V + caches.K_exp + caches.V_exp)
        assert all(int((t != 0).sum()) > 0 for t in got[-1])
    for a, b in zip(*got):
        assert torch.equal(a, b)
