"""Attention over the 4-bit cache where queries of one tile see different
positions: each row's result is its own.  The cache, the definition in 64 bits
and its derived tolerance are those of tests/test_gpu_kv4.py."""
import pytest

from tests.test_gpu_kv4 import Sequences, _attend, env  # noqa: F401  (env: the fixture)

pytestmark = pytest.mark.gpu

# (positions, new tokens, query heads, key heads, window, tokens that are checked): the
# single-token kernel, a wavefront's tiles eight apart, the window's lower edges on
# both sides of a tile's end; the chunk kernel, tiles one after another
WINDOWED = {"few": (700, 16, 1, 1, 334, None), "chunk": (400, 300, 96, 96, 50, [0, 1, 5, 18, 19, 31, 32, 150, 298, 299])}


@pytest.mark.parametrize("which", list(WINDOWED))
@pytest.mark.parametrize("tiny", ["scale", "queries"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_vanish_under_a_window(env, which, tiny, D):  # noqa: F811
    """A query whose window opens in a later tile than its neighbours': the mean
    of what it sees, as for them."""
    torch, _ = env
    n, m, heads, kv_heads, window, only = WINDOWED[which]
    s = Sequences(env, [n], [m], kv_heads, D, 32, "bfloat16", seed=31)
    s.fill()
    q = torch.randn(m, heads, D, generator=s.g, device="cuda")
    q = (q * 2.0 ** -115 if tiny == "queries" else q).to(s.dtype)
    assert (q != 0).any(-1).all()
    _attend(env, s, heads, window=window, q=q, scale=2.0 ** -120 if tiny == "scale" else None, only=only)


@pytest.mark.parametrize("length", [-1, -100, -(2 ** 31) + 5, -(2 ** 31)])
@pytest.mark.parametrize("shape", [(16, 4, 2), (300, 96, 96)], ids=str)
def test_lengths_below_zero(env, length, shape):  # noqa: F811
    """A sequence of less than no positions: nothing is written, gathered or seen."""
    torch, celty = env
    n, heads, kv_heads = shape
    s = Sequences(env, [n], [n], kv_heads, 64, 32, "float16", seed=32)
    s.append()
    before = s.arrays()
    s.kv_len.fill_(length)
    q = torch.randn(n, heads, 64, generator=s.g, device="cuda").half()
    for seqs, t in ((s.seqs, n), (celty.Kv4Seqs(s.table, s.kv_len), 1)):
        out = torch.full_like(q[:t], float("nan"))
        celty.celty_kv4_attention(s.cache, seqs, q[:t], out, celty.new_kv4_workspace(s.cache, seqs, t, heads))
        assert (out == 0).all()
        k, v = torch.full_like(s.k[0][:t], 3.0), torch.full_like(s.v[0][:t], 3.0)
        celty.celty_kv4_append(s.cache, seqs, k, v)
        celty.celty_kv4_gather(s.cache, seqs, k, v)
        assert (k == 0).all() and (v == 0).all()
    for a, b in zip(s.arrays(), before):
        assert (a.view("u1") == b.view("u1")).all()
