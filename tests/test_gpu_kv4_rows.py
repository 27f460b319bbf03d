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
