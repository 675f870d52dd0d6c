"""The embedding's gradient where only large inputs reach: several tiles of steps in a
workgroup of the sort (more than 131072 steps), and pieces of 64, 128 and 256 steps (more
than 131072, 262144 and 524288 steps times blocks of 512 columns), summed by whole waves
and by parts of one.

dy holds whole numbers within 8 and every row's sum stays below 2^24, so sums are exact in
any order: equal to the bit, and rounded once where the table is bf16."""
import pytest

from test_gpu_embedding import TYPES, _tokens

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,V,D,kind", [
    # 2 to 5 tiles a workgroup: one, two and three passes of digits
    (131073, 300, 8, "zipf"), (131073, 50000, 8, "zipf"), (140001, 7, 3, "outside"),
    (262145, 9, 16, "one"), (300007, 300, 24, "zipf"), (300007, 70000, 5, "even"),
    (270001, 2 ** 22 + 3, 2, "zipf"), (524289 + 4000, 2000, 4, "outside"), (300007, 40, 130, "none"),
    # pieces of 64, 128 and 256: narrow rows, a whole wave's, several blocks of columns
    (140001, 5000, 64, "zipf"), (300007, 12, 200, "outside"), (600011, 300, 33, "zipf"),
    (140001, 900, 300, "zipf"), (300007, 3, 264, "even"), (600011, 30, 300, "zipf"),
    (70003, 400, 520, "zipf"), (140001, 2, 520, "one"), (300007, 1000, 520, "outside"),
    (300007, 100, 513, "zipf"), (60001, 50, 2050, "zipf"), (120001, 700, 2560, "zipf")])
def test_whole_numbers(sw, T, V, D, kind, types):
    print("case embedding many", T, V, D, kind, types, flush=True)
    tdt, ydt = (TYPES[n] for n in types)
    tokens = torch.from_numpy(_tokens(kind, T, V, T + V)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(T + D)
    dy = torch.randint(-8, 9, (T, D), generator=gen, device="cuda", dtype=torch.int8)
    want = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    there = (tokens >= 0) & (tokens < V)
    want.index_add_(0, tokens[there], dy[there].double())
    assert want.abs().max() < 2 ** 24
    got = sw.embedding_bwd(tokens, dy.to(ydt), V, dtype=tdt)
    assert torch.equal(got, want.float().to(tdt))
    # int32 tokens, rows of a wider tensor, a scale that is exact
    wide = torch.zeros(T, D + 3, device="cuda", dtype=ydt)
    wide[:, 1:1 + D] = dy
    got = sw.embedding_bwd(tokens.clamp(-1, 2 ** 31 - 1).to(torch.int32), wide[:, 1:1 + D], V, dtype=tdt, scale=-0.5)
    assert torch.equal(got, (want.float() * -0.5).to(tdt))
