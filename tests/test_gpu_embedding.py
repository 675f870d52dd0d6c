"""The scaled embedding and its table's gradient against their 64-bit definitions.

Tolerances: a row is one product rounded to fp32 (and once more to bf16, 2^-8); a gradient
of n terms is off by at most n + 2 roundings of 2^-24 of the terms' sum, in any order, and
2^-8 of the value more in bf16."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _near(got, want, most, what):
    g = got.double().cpu().numpy()
    most = most + 1e-38
    if got.dtype is torch.bfloat16:
        most = most * 1.01 + 2.0 ** -8 * np.abs(want)
    err = np.abs(g - want)
    assert (err <= most).all(), f"{what}: {np.max(err / most):.3g} of the bound"


def _tokens(kind, T, V, seed):
    g = np.random.Generator(np.random.PCG64(seed))
    if kind == "even":
        t = g.integers(0, V, T)
    elif kind == "zipf":
        t = np.minimum(np.exp(g.random(T) * np.log(V + 1)).astype(np.int64) - 1, V - 1)
        t = g.permutation(V)[t]
    elif kind == "one":
        t = np.full(T, V // 2)
    elif kind == "each":
        t = np.arange(T) % V
    elif kind == "none":
        t = np.where(np.arange(T) % 2, -1, V)
    else:  # some of no row, far outside
        t = g.integers(0, V, T)
        t[::3] = -1
        t[1::7] = V
        t[2::11] = 2 ** 31 - 1
    return t


def _check(sw, tokens, V, D, types, scale, wide):
    tdt, ydt = (TYPES[n] for n in types)
    T = len(tokens)
    g = np.random.Generator(np.random.PCG64(T + V + D))
    table = torch.from_numpy(g.standard_normal((V, D))).to(tdt)
    dy = torch.from_numpy(g.standard_normal((T, D))).to(ydt)
    tok = torch.from_numpy(tokens).to(torch.int64 if wide else torch.int32).cuda()
    there = (tokens >= 0) & (tokens < V)
    s = float(np.float32(scale))
    want = np.where(there[:, None], table.double().numpy()[np.where(there, tokens, 0)] * s, 0.0)
    leaf = table.cuda().requires_grad_(True)
    y = sw.embedding_fn(tok, leaf, scale=scale, dtype=ydt)
    assert y.dtype is ydt and y.shape == (T, D)
    _near(y.detach(), want, 2.0 ** -24 * np.abs(want), "y")
    assert torch.equal(y, sw.embedding_fwd(tok, table.cuda(), scale=scale, dtype=ydt))
    (got,) = torch.autograd.grad(y, leaf, dy.cuda())
    assert got.dtype is tdt
    d = dy.double().numpy()
    total, size, count = np.zeros((V, D)), np.zeros((V, D)), np.zeros(V)
    np.add.at(total, tokens[there], d[there])
    np.add.at(size, tokens[there], np.abs(d[there]))
    np.add.at(count, tokens[there], 1)
    _near(got, s * total, abs(s) * size * (count[:, None] + 2) * 2.0 ** -24, "dtable")
    assert (got[torch.from_numpy(count == 0).cuda()] == 0).all()
    assert torch.equal(got, sw.embedding_bwd(tok, dy.cuda(), V, scale=scale, dtype=tdt))


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,V,D,kind", [
    (1, 1, 1, "even"), (1, 50, 8, "even"), (2, 3, 7, "even"), (17, 5, 33, "zipf"), (64, 1000, 64, "even"),
    (300, 7, 65, "zipf"), (1000, 256, 128, "zipf"), (777, 5000, 96, "outside"), (2048, 100, 40, "one"),
    (2049, 3000, 24, "each"), (100, 40, 16, "none"), (5000, 70000, 16, "zipf"), (4097, 2, 256, "even"),
    (3000, 300, 520, "zipf"), (40, 30, 2050, "even"),
    # the last and first sizes of the sorts in one launch and by digits
    (63, 9, 8, "outside"), (65, 9, 8, "one"), (4096, 300, 24, "zipf"), (4097, 300, 24, "outside"),
    (8191, 5000, 16, "outside"), (8192, 5000, 24, "one"), (8193, 5000, 24, "zipf")])
def test_values_and_gradients(sw, T, V, D, kind, types):
    print("case embedding", T, V, D, kind, types, flush=True)
    _check(sw, _tokens(kind, T, V, T + V), V, D, types, [1.0, 0.37, -22.6][T % 3], T % 2 == 0)


@pytest.mark.parametrize("T,V,D,kind", [(40000, 30, 12, "zipf"), (70001, 300000, 4, "zipf"), (66000, 5, 8, "one"),
                                        (30000, 2 ** 22 + 3, 2, "even"), (20000, 65536, 8, "outside")])
def test_many_tokens(sw, T, V, D, kind):
    print("case embedding", T, V, D, kind, flush=True)
    _check(sw, _tokens(kind, T, V, T), V, D, ("f32", "f32"), 2.0, T % 2 == 0)


def test_sums_keep_to_their_rows(sw):
    """Whole numbers, whose sums are exact: equal to the bit, in every row, over tiles and
    sequences of all kinds."""
    g = np.random.Generator(np.random.PCG64(1))
    for T, V, D in ((8191, 3, 9), (8192, 4000, 8), (12345, 50, 72), (100000, 1000, 3)):
        tokens = np.sort(_tokens("zipf", T, V, T)) if T % 2 else _tokens("zipf", T, V, T)
        dy = g.integers(-8, 9, (T, D))
        want = np.zeros((V, D), dtype=np.int64)
        np.add.at(want, tokens, dy)
        got = sw.embedding_bwd(torch.from_numpy(tokens).cuda(), torch.from_numpy(dy).float().cuda(), V)
        assert np.array_equal(got.cpu().numpy().astype(np.int64), want), (T, V, D)


def test_shapes_strides_and_what_is_not_finite(sw):
    V, D = 60, 48
    table = torch.randn(V, D, device="cuda")
    tok = torch.randint(0, V, (3, 5, 7), device="cuda")
    y = sw.embedding_fwd(tok, table)
    assert y.shape == (3, 5, 7, D) and torch.equal(y, table[tok])
    wide = torch.randn(3, 5, 7, 2 * D + 1, device="cuda")
    for dy in (wide[..., :D], wide[..., 1:1 + D], wide[..., :D].transpose(0, 1).contiguous().transpose(0, 1),
               torch.randn(1, 1, 1, D, device="cuda").expand(3, 5, 7, D)):
        a = sw.embedding_bwd(tok, dy, V, dtype=torch.float32)
        assert torch.equal(a, sw.embedding_bwd(tok, dy.contiguous(), V, dtype=torch.float32))
    # a row that is not finite, and a gradient that is not, reach their own rows only;
    # of padding neither is read
    table[9] = float("nan")
    t = torch.tensor([8, 9, 10, -1, 8], device="cuda")
    y = sw.embedding_fwd(t, table)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2, 3, 4]]).all() and (y[3] == 0).all()
    dy = torch.randn(5, D, device="cuda")
    dy[3] = float("nan")
    dy[1, 5] = float("inf")
    g = sw.embedding_bwd(t, dy, V)
    assert torch.isinf(g[9, 5]) and torch.isfinite(g).sum() == V * D - 1


def test_no_tokens_no_rows(sw):
    for kind in (torch.int32, torch.int64):
        none = torch.empty(0, dtype=kind, device="cuda")
        table = torch.randn(9, 16, device="cuda")
        assert sw.embedding_fwd(none, table).shape == (0, 16)
        assert torch.equal(sw.embedding_bwd(none, torch.empty(0, 16, device="cuda"), 9), torch.zeros_like(table))
        some = torch.zeros(4, dtype=kind, device="cuda")
        assert (sw.embedding_fwd(some, table[:0]) == 0).all()
        assert sw.embedding_bwd(some, torch.randn(4, 16, device="cuda"), 0).shape == (0, 16)
        assert sw.embedding_fwd(some, table[:, :0]).shape == (4, 0)
        assert sw.embedding_bwd(some, torch.empty(4, 0, device="cuda"), 9).shape == (9, 0)


def test_graphs_and_streams(sw):
    V, D, T = 3000, 64, 5000
    table = torch.randn(V, D, device="cuda")
    tok = torch.from_numpy(_tokens("zipf", T, V, 3)).cuda()
    dy = torch.randn(T, D, device="cuda").bfloat16()

    def work():
        return sw.embedding_fwd(tok, table, scale=3.0), sw.embedding_bwd(tok, dy, V, scale=3.0)

    work()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = work()
        graphs.append((graph, outs))
    for i in range(3):
        tok.copy_(torch.from_numpy(_tokens("zipf" if i else "outside", T, V, 10 + i)))
        for graph, outs in graphs:
            graph.replay()
            torch.cuda.synchronize()
            kept = [o.clone() for o in outs]
            assert all(torch.equal(a, b) for a, b in zip(kept, work())), i
    want = work()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(3):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(work())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for one in got for a, b in zip(one, want))


def test_offsets_past_32_bits(sw):
    """A table and rows whose bytes and elements pass 2^32."""
    V, D = 2 ** 21 + 5, 1100
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    tok = torch.tensor([V - 1, 0, V - 2, V - 1], device="cuda")
    table[-2:] = torch.randn(2, D, device="cuda").bfloat16()
    assert torch.equal(sw.embedding_fwd(tok, table), table[tok])
    dy = torch.randn(4, D, device="cuda").bfloat16()
    del table
    g = sw.embedding_bwd(tok, dy, V)
    assert torch.equal(g[V - 2], dy[2]) and torch.equal(g[0], dy[1])
    assert torch.equal(g[V - 1], (dy[0].float() + dy[3].float()).bfloat16())
    assert (g[1:V - 2] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tables_and_workspaces_off_16_bytes(sw, dtype):
    """Through the C ABI: a gradient at any address of its type's alignment, its neighbours
    untouched; a workspace too small is refused."""
    from paper_2606_00601_amd._bind import _on
    dt, code = TYPES[dtype], 0 if dtype == "f32" else 1
    f = sw.fast()
    for V, D, off in ((1, 1, 1), (3, 2, 1), (5, 7, 3), (40, 24, 5), (300, 33, 7)):
        tok = torch.randint(0, V, (50,), device="cuda")
        dy = torch.randn(50, D, device="cuda").to(dt)
        want = sw.embedding_bwd(tok, dy, V)
        buf = torch.full((V * D + 32,), 7.0, device="cuda", dtype=dt)
        out = buf[off:off + V * D]
        n = f.sw_embedding_bwd_workspace(50, V, D)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        with _on(tok.device):
            args = (tok.data_ptr(), dy.data_ptr(), out.data_ptr(), 50, V, D, D, code, code, 1, 1.0)
            assert f.sw_embedding_bwd(*args, ws.data_ptr(), n - 1) == 1
            assert f.sw_embedding_bwd(*args, ws.data_ptr(), n) == 0
        assert torch.equal(out.view(V, D), want)
        assert (buf[:off] == 7.0).all() and (buf[off + V * D:] == 7.0).all()
        with _on(tok.device):  # from the pool
            out.fill_(7.0)
            assert f.sw_embedding_bwd(*args, None, 0) == 0
        assert torch.equal(out.view(V, D), want)


def test_refusals(sw):
    table = torch.randn(9, 16, device="cuda")
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    dy = torch.randn(4, 16, device="cuda")
    for bad in (tok.float(), tok.to(torch.int16)):
        with pytest.raises(TypeError):
            sw.embedding_fwd(bad, table)
    with pytest.raises(ValueError):
        sw.embedding_fwd(tok.cpu(), table)
    with pytest.raises(ValueError):
        sw.embedding_fwd(torch.zeros(8, dtype=torch.int64, device="cuda")[::2], table)
    with pytest.raises(TypeError):
        sw.embedding_fwd(tok, table.half())
    with pytest.raises(TypeError):
        sw.embedding_fwd(tok, table, dtype=torch.float16)
    with pytest.raises(ValueError):
        sw.embedding_fwd(tok, table.t())
    with pytest.raises(ValueError):
        sw.embedding_bwd(tok, dy[:3], 9)
    with pytest.raises(TypeError):
        sw.embedding_bwd(tok, dy.half(), 9)
    with pytest.raises(ValueError):
        sw.embedding_bwd(tok, torch.randn(16, 4, device="cuda").t(), 9)
