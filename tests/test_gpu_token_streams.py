"""The head norm and the embedding on several streams and from two host threads at once,
each with inputs and sizes of its own, so that scratch shared by mistake would show: the
bits of the same calls one after the other.  With a workspace from the Python functions
and, through the C ABI, from the stream-ordered pool."""
import threading

import pytest

from test_gpu_embedding import _tokens

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _embedding(sw, j, pool):
    """A call's work on inputs of its own: many steps (by digits), few (by counting)."""
    from paper_2606_00601_amd._bind import _on
    T, V, D = [(9000, 3000, 64), (20011, 700, 96), (4000, 5000, 200), (15000, 40, 33)][j]
    gen = torch.Generator(device="cuda").manual_seed(j)
    tok = torch.from_numpy(_tokens("zipf", T, V, j)).cuda()
    dy = torch.randn(T, D, generator=gen, device="cuda")
    table = torch.randn(V, D, generator=gen, device="cuda")

    def work():
        y = sw.embedding_fwd(tok, table, scale=3.0)
        if not pool:
            return [y, sw.embedding_bwd(tok, dy, V, scale=3.0)]
        g = torch.empty(V, D, device="cuda")
        with _on(g.device):
            assert sw.fast().sw_embedding_bwd(tok.data_ptr(), dy.data_ptr(), g.data_ptr(), T, V, D, D, 0, 0, 1,
                                              3.0, None, 0) == 0
        return [y, g]

    return work


def _head_norm(sw, j, pool):
    from paper_2606_00601_amd._bind import _on
    B, L, H, Hk, K = [(2, 700, 6, 2, 64), (1, 3001, 4, 4, 32), (3, 333, 12, 3, 128), (2, 1500, 5, 1, 40)][j]
    gen = torch.Generator(device="cuda").manual_seed(10 + j)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, dq, dk = (make(B, L, n, K) for n in (H, Hk, H, Hk))
    w = [torch.rand(K, generator=gen, device="cuda") + 0.5 for _ in "qk"]
    how = dict(inv_freq=torch.rand(K // 4, generator=gen, device="cuda"))
    R = 2 * (K // 4)

    def work():
        y = sw.head_norm_fwd(q, k, *w, **how)
        if not pool:
            return [*y, *sw.head_norm_bwd(dq, dk, q, k, *w, **how).values()]
        g = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(w[0]), torch.empty_like(w[1])]
        st = ((L * H * K, H * K, K) + (L * Hk * K, Hk * K, K)) * 2 + (0, 0)
        with _on(q.device):
            assert sw.fast().sw_head_norm_bwd(
                *(t.data_ptr() for t in (dq, dk, q, k, *w)), None, how["inv_freq"].data_ptr(),
                *(t.data_ptr() for t in g), B, L, H, Hk, K, R, st, 1, 0, 1e-6, None, 0) == 0
        return [*y, *g]

    return work


@pytest.mark.parametrize("pool", [False, True])
@pytest.mark.parametrize("make", [_embedding, _head_norm])
def test_streams(sw, make, pool):
    works = [make(sw, j, pool) for j in range(4)]
    want = [w() for w in works]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in works]
    for turn in range(4):
        got = []
        for j in range(len(works)):
            with torch.cuda.stream(streams[(j + turn) % len(streams)]):
                got.append(works[j]())
        torch.cuda.synchronize()
        for j, (a, b) in enumerate(zip(got, want)):
            assert all(torch.equal(p, q) for p, q in zip(a, b)), (turn, j)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("pool", [False, True])
@pytest.mark.parametrize("make", [_embedding, _head_norm])
def test_two_threads(sw, make, pool, shared):
    """On streams of their own and on one of both."""
    works = [make(sw, j, pool) for j in range(2)]
    want = [w() for w in works]
    torch.cuda.synchronize()
    both, errors = torch.cuda.Stream(), []

    def worker(j):
        try:
            stream = both if shared else torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    got = works[j]()
                    stream.synchronize()
                    if not all(torch.equal(p, q) for p, q in zip(got, want[j])):
                        errors.append(f"thread {j} differs")
        except Exception as e:  # reported below
            errors.append(f"thread {j}: {e!r}")

    threads = [threading.Thread(target=worker, args=(j,)) for j in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    assert not any(t.is_alive() for t in threads) and not errors, errors
