"""Every position that a token sees counts once, and no other: with equal scores
the result is the mean of the values seen.  All values are zero but one a head,
so a result is that value over the number of positions, or zero.

Tolerance: that of tests/test_gpu_kv4.py where scores are exact (all keys are
zero) and one value of weight 1 / n is not zero: the output's rounding, and
2^-10 + 2^-20 of twice that value's share for its probability, which is rounded
with the value's scale.  A value that is not seen leaves zeros, exactly."""
import numpy as np
import pytest

from tests.test_gpu_kv4 import UNIT, Sequences, _expect, env  # noqa: F401

pytestmark = pytest.mark.gpu


class Marked:
    """One sequence whose keys and values are zeros; mark() sets one value a head."""

    def __init__(self, env, n, kv_heads, D, page, seed):  # noqa: F811
        torch, celty = self.env = env
        pages = -(-n // page) + 1   # one beyond the sequence's last
        self.n, self.H, self.D, self.page = n, kv_heads, D, page
        self.cache = celty.Kv4Cache(pages, kv_heads, D, page)
        self.table = torch.from_numpy(np.random.default_rng(seed).permutation(pages).astype(np.int32)).cuda().view(1, -1)
        self.kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
        # 0 and 15 steps of 546, exact in fp16, in alternating channels
        self.value = torch.zeros(D, device="cuda", dtype=torch.float16)
        self.value[1::2] = 8190.0

    def mark(self, positions, on=True):
        """Head h's value at positions[h]; several heads may share one."""
        torch, celty = self.env
        for j in sorted(set(positions)):
            v = torch.zeros(1, self.H, self.D, dtype=torch.float16, device="cuda")
            if on:
                for h, p in enumerate(positions):
                    if p == j:
                        v[0, h] = self.value
            at = celty.Kv4Seqs(self.table, torch.tensor([j + 1], dtype=torch.int32, device="cuda"))
            celty.celty_kv4_append(self.cache, at, torch.zeros_like(v), v)

    def check(self, m, group, window, positions, stored=None):
        """m new tokens of `group` query heads a key head, positions[h] marked."""
        torch, celty = self.env
        heads = self.H * group
        start = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        seqs = celty.Kv4Seqs(self.table, self.kv_len, start if m > 1 else None)
        q = torch.ones(m, heads, self.D, dtype=torch.float16, device="cuda")
        out = torch.full_like(q, float("nan"))
        self.mark(positions)
        celty.celty_kv4_attention(self.cache, seqs, q, out, celty.new_kv4_workspace(self.cache, seqs, m, heads), window=window)
        self.mark(positions, on=False)
        stored = np.ones(self.n, bool) if stored is None else stored
        before = np.concatenate([[0], np.cumsum(stored)])
        last = np.arange(self.n - m, self.n)
        first = np.maximum(0, last - window + 1) if window else np.zeros_like(last)
        count = before[last + 1] - before[first]
        j = np.array(positions)
        seen = (j[None] >= first[:, None]) & (j[None] <= last[:, None])
        seen &= np.array([j_ < self.n and stored[j_] for j_ in positions])[None]
        want = np.where(seen, 8190.0 / np.maximum(count, 1)[:, None], 0.0)
        got = out.double().cpu().numpy().reshape(m, self.H, group, self.D)
        want = np.broadcast_to(want[:, :, None, None], got.shape)
        share = (2.0 ** -10 + 2.0 ** -20) * 2 * want
        bad = np.abs(got[..., 0::2]) > share[..., 0::2]
        bad |= ~(np.abs(got[..., 1::2] - want[..., 1::2]) <= 2.0 ** -11 * want[..., 1::2] + share[..., 1::2])
        assert not bad.any(), [(int(i), positions[h], got[i, h, 0, 1], want[i, h, 0, 1]) for i, h in np.argwhere(bad.any((2, 3)))[:5]]


def _positions(n, extra, count, seed):
    """Ends of octets, tiles, pages and long stretches, the sequence's own ends, the
    one behind it, and others."""
    rng = np.random.default_rng(seed)
    p = {0, 1, 7, 8, 31, 32, 33, 63, 64, 255, 256, 511, 512, 513, n // 2, n - 33, n - 32, n - 31, n - 2, n - 1, n}
    p |= {512 * i + d for i in range(1, n // 512 + 1) for d in (-1, 0)} if n < 3000 else {4096 * i + d for i in range(1, n // 4096 + 1) for d in (-1, 0)}
    p |= set(extra)
    p = sorted(j for j in p if 0 <= j <= n)
    return p + [int(j) for j in rng.integers(0, n, max(0, count - len(p)))]


@pytest.mark.parametrize("n", [1, 33, 64, 513, 1000, 5001, 20011])
@pytest.mark.parametrize("m,group", [(1, 1), (1, 5), (7, 3), (40, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_each_position_counts_once(env, n, m, group, D):  # noqa: F811
    if m > n:
        m = n
    s = Marked(env, n, 8, D, 64 if n % 2 else 32, seed=n + m)
    p = _positions(n, [n - m - 1, n - m, n - m + 1], 48, n)
    for i in range(0, len(p), 8):
        s.check(m, group, 0, (p[i:i + 8] * 8)[:8])


@pytest.mark.parametrize("n,window", [(64, 1), (700, 40), (5001, 334), (20011, 4000), (20011, 16385)])
@pytest.mark.parametrize("m,group", [(1, 4), (9, 2), (16, 1)])
def test_each_position_of_a_window_counts_once(env, n, window, m, group):  # noqa: F811
    s = Marked(env, n, 8, 64, 32, seed=window)
    first = n - m - window + 1
    p = _positions(n, [j for d in (-33, -32, -1, 0, 1, m - 2, m - 1, m, 31, 32) if 0 <= (j := first + d) < n], 40, n)
    for i in range(0, len(p), 8):
        s.check(m, group, window, (p[i:i + 8] * 8)[:8])


@pytest.mark.parametrize("n,m,window", [(9000, 400, 0), (9000, 400, 333), (20011, 300, 0), (700, 700, 0), (700, 650, 50)])
@pytest.mark.parametrize("D", [64, 128])
def test_each_position_of_a_chunk_counts_once(env, n, m, window, D):  # noqa: F811
    """The chunk kernel, its contexts shared by several workgroups among them."""
    H = 64
    s = Marked(env, n, H, D, 64, seed=m)
    extra = [n - m - 1, n - m, n - m + 1, n - m + 127, n - m + 128, 8191, 8192, 8193]
    extra += [j for d in (-1, 0, 1, 31, 32) if 0 <= (j := n - m - window + 1 + d) < n]
    p = _positions(n, [j for j in extra if 0 <= j < n], 2 * H, n + m)
    for i in range(0, 2 * H, H):
        s.check(m, 1, window, (p[i:i + H] * H)[:H])


@pytest.mark.parametrize("m,H", [(1, 8), (24, 8), (400, 64)])
def test_positions_of_hidden_pages_do_not_count(env, m, H):  # noqa: F811
    """Missing pages at the ends of the workgroups' shares and in the middle of them."""
    torch, _ = env
    n, page = 9000, 64
    s = Marked(env, n, H, 64, page, seed=m)
    stored = np.ones(n, bool)
    hidden = [0, 7, 8, 70, 127, 128]
    marks = [p * page + d for p in hidden for d in (-1, 0, 31, 32, 63, 64) if 0 <= p * page + d < n]
    marks += [n - 1, n - 2]
    marks = (marks * H)[:H * -(-len(marks) // H)]
    for p in hidden:
        stored[p * page:(p + 1) * page] = False
    table = s.table.clone()
    hole = table.clone()
    for p, bad in zip(hidden, [-1, 10 ** 6, -1, -(2 ** 31), 2 ** 31 - 1, -7]):
        hole[0, p] = bad
    for i in range(0, len(marks), H):
        mine = marks[i:i + H]
        s.table = table
        s.mark(mine)          # the pages hold the values, the table does not name them
        s.table = hole
        s.check(m, 1, 0, mine, stored)
        s.table = table
        s.mark(mine, on=False)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n,m,heads,kv_heads,D,window,only", [
    (1000, 1, 8, 2, 128, 0, None), (5001, 1, 8, 2, 64, 0, None), (20011, 1, 8, 2, 128, 0, None), (20011, 5, 6, 2, 64, 4000, None),
    (9000, 400, 64, 64, 64, 0, [0, 1, 200, 399]), (9000, 400, 64, 64, 128, 2000, [0, 127, 128, 399])])
def test_error_in_norm(env, dtype, n, m, heads, kv_heads, D, window, only):  # noqa: F811
    """Over a row of D channels of random values the roundings do not add up: the
    output's is at most its unit u in norm.  A probability's is 2^-11 at most, of
    n independent terms whose sum in squares is about the output's square, for
    values of random sign: another 2^-11 in norm; a bias in the values adds to the
    output alone.  Half as much again for rows with a small norm by chance.  One
    position more or less of 20011 changes the norm by 2^-7."""
    torch, celty = env
    s = Sequences(env, [n], [m], kv_heads, D, 64, dtype, seed=n + m)
    s.fill()
    q = torch.randn(m, heads, D, generator=s.g, device="cuda").to(s.dtype)
    out = torch.full_like(q, float("nan"))
    celty.celty_kv4_attention(s.cache, s.seqs, q, out, celty.new_kv4_workspace(s.cache, s.seqs, m, heads), window=window)
    want, _ = _expect(s, q, heads, D ** -0.5, window, only=only)
    got = out.double().cpu().numpy()
    got = got if only is None else got[only]
    error = np.linalg.norm(got - want, axis=2) / np.linalg.norm(want, axis=2)
    assert error.max() <= 1.5 * (UNIT[dtype] + 2.0 ** -11), error.max()
