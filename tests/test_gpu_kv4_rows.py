"""Attention over the 4-bit cache where queries of one tile see different
positions: each row's result is its own.  The cache, the definition in 64 bits
and its derived tolerance are those of tests/test_gpu_kv4.py."""
import numpy as np
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


def _set_params(torch, s, first, last, scale, minimum):
    """Key and value parameters of positions first..last-1 of the one sequence."""
    t = torch.arange(first, last, device="cuda")
    pages, slots = s.table[0].long()[t // s.page], t % s.page
    p = torch.tensor([scale, minimum], device="cuda").half()
    for x in (s.cache.k_params, s.cache.v_params):
        x[pages, :, slots] = p


@pytest.mark.parametrize("which", list(WINDOWED))
@pytest.mark.parametrize("scale", [float("inf"), 65504.0, float("nan"), float("-inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_positions_before_every_window_do_not_matter(env, which, scale, D):  # noqa: F811
    """A caller that keeps the last `window` tokens only: whatever is in the
    memory of the others, the results are the same bits."""
    torch, celty = env
    n, m, heads, kv_heads, window, only = WINDOWED[which]
    s = Sequences(env, [n], [m], kv_heads, D, 32, "float16", seed=33, ranges=(1.0, 2.0 ** -8))
    s.fill()
    q, out, ws = _attend(env, s, heads, window=window, only=only)
    first = n - m - window + 1
    assert first > 0
    _set_params(torch, s, 0, first, scale, 1.0)
    got = torch.full_like(out, float("nan"))
    celty.celty_kv4_attention(s.cache, s.seqs, q, got, ws, window=window)
    assert torch.equal(got, out)


@pytest.mark.parametrize("which", list(WINDOWED))
@pytest.mark.parametrize("window", [True, False])
def test_later_tokens_do_not_matter(env, which, window):  # noqa: F811
    """A token's result is the same bits whatever the tokens after it hold,
    values far above its own among them."""
    torch, celty = env
    n, m, heads, kv_heads, w, only = WINDOWED[which]
    w = w if window else 0
    s = Sequences(env, [n], [m], kv_heads, 64, 32, "float16", seed=34, ranges=(1.0, 2.0 ** -8))
    s.fill()
    q, out, ws = _attend(env, s, heads, window=w, only=only)
    for keep in (1, m // 2, m - 1):   # tokens of the call
        a = n - m + keep
        s.v[0][a:] = 20000.0 * torch.randn(n - a, kv_heads, 64, generator=s.g, device="cuda").clamp(-3, 3).half()
        s.k[0][a:] *= 8.0
        s.append()
        got = torch.full_like(out, float("nan"))
        celty.celty_kv4_attention(s.cache, s.seqs, q, got, ws, window=w)
        assert torch.equal(got[:keep], out[:keep]), keep
        s = Sequences(env, [n], [m], kv_heads, 64, 32, "float16", seed=34, ranges=(1.0, 2.0 ** -8))
        s.fill()


LARGE = {"products": (1.0, 2.0 ** 13, None), "scale": (1.0, 1.0, 1e30), "largest_scale": (1.0, 1.0, 3.4e38),
         "negative_scale": (1.0, 1.0, -1e12), "queries": (2.0 ** 118, 1.0, None), "queries_small_scale": (2.0 ** 124, 1.0, 2.0 ** -90)}


@pytest.mark.parametrize("case", list(LARGE))
@pytest.mark.parametrize("which", ["one", "split"] + list(WINDOWED))
def test_scores_far_apart(env, case, which):  # noqa: F811
    """Scores in the millions and far beyond: all of the weight is with the largest,
    however little of it a step of fp32 there leaves to an exponential.  Rows whose
    two largest are nearer than what the scores' sums may err by are left out:
    (D + 8) 2^-24 of the largest sum of magnitudes, twice."""
    torch, celty = env
    q_range, k_range, scale = LARGE[case]
    D = 64
    n, m, heads, kv_heads, window, only = dict(one=(300, 1, 2, 1, 0, None), split=(9000, 1, 2, 1, 0, None), **WINDOWED)[which]
    if case == "products":
        q_range = 2.0 ** 13
    s = Sequences(env, [n], [m], kv_heads, D, 32, "bfloat16", seed=35, ranges=(k_range, 1.0))
    s.fill()
    q = (torch.randn(m, heads, D, generator=s.g, device="cuda") * q_range).to(s.dtype)
    assert q.isfinite().all()
    out = torch.full_like(q, float("nan"))
    celty.celty_kv4_attention(s.cache, s.seqs, q, out, celty.new_kv4_workspace(s.cache, s.seqs, m, heads), scale=scale, window=window)
    assert out.isfinite().all()
    k, v = s.values(0)
    sign = -1.0 if scale is not None and scale < 0 else 1.0
    factor = abs(scale) if scale is not None else D ** -0.5
    checked = 0
    for i in only if only is not None else range(m):
        last = n - m + i
        first = max(0, last - window + 1) if window else 0
        for h in range(0, heads, 5):
            g = h * kv_heads // heads
            x = q[i, h].double().cpu().numpy()
            z = sign * (k[first:last + 1, g] @ x)
            order = np.argsort(z)
            room = 2 * (D + 8) * 2.0 ** -24 * 2 * np.abs(x).sum() * np.abs(k[first:last + 1, g]).max()
            if len(z) > 1 and (z[order[-1]] - z[order[-2]] <= room or (z[order[-1]] - z[order[-2]] - room) * factor < 30):
                continue
            checked += 1
            want = v[first + order[-1], g]
            # a probability of one: its rounding with the value's scale, and the output's
            assert (np.abs(out[i, h].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * np.abs(want).max()).all(), (i, h)
    assert checked > 0


@pytest.mark.parametrize("which", ["one"] + list(WINDOWED))
@pytest.mark.parametrize("bad", [float("-inf"), float("inf"), float("nan")])
@pytest.mark.parametrize("positive", [True, False])
def test_queries_that_are_not_finite(env, which, bad, positive):  # noqa: F811
    """No softmax is left of scores of infinity: NaN, whatever their sign, and in
    the query's own row alone."""
    torch, celty = env
    n, m, heads, kv_heads, window, only = dict(one=(300, 1, 2, 1, 0, None), **WINDOWED)[which]
    s = Sequences(env, [n], [m], kv_heads, 64, 32, "float16", seed=36)
    if positive:   # every minimum and every code of channel 5 above zero
        s.k[0] = s.k[0].abs() + 1.0
        s.k[0][:, :, 5] += 9.0
    s.fill()
    q, out, ws = _attend(env, s, heads, window=window, only=only)
    row, h = m - 1, heads - 1
    q[row, h, 5] = bad
    got = torch.zeros_like(out)
    celty.celty_kv4_attention(s.cache, s.seqs, q, got, ws, window=window)
    assert got[row, h].isnan().all()
    got[row, h] = out[row, h]
    assert torch.equal(got, out)


def test_queries_and_results_beside_each_other(env):  # noqa: F811
    """One tensor that holds both: whole heads side by side, and head by head."""
    torch, celty = env
    s = Sequences(env, [70, 33], [20, 3], 2, 64, 32, "float16", seed=37)
    s.fill()
    q, out, ws = _attend(env, s, 4)
    for shape, parts in (((23, 8, 64), lambda t: (t[:, :4], t[:, 4:])), ((23, 4, 2, 64), lambda t: (t[:, :, 0], t[:, :, 1])),
                         ((4, 23, 2, 64), lambda t: (t[:, :, 0].permute(1, 0, 2), t[:, :, 1].permute(1, 0, 2)))):
        both = torch.full(shape, 7.0, dtype=torch.float16, device="cuda")
        qv, ov = parts(both)
        qv.copy_(q)
        celty.celty_kv4_attention(s.cache, s.seqs, qv, ov, ws)
        assert torch.equal(ov, out) and torch.equal(qv, q)
    kv = torch.empty(23, 2, 2, 64, dtype=torch.float16, device="cuda")
    celty.celty_kv4_gather(s.cache, s.seqs, kv[:, 0], kv[:, 1])
    k, v = torch.empty_like(kv[:, 0]), torch.empty_like(kv[:, 0])
    celty.celty_kv4_gather(s.cache, s.seqs, k, v)
    assert torch.equal(kv[:, 0], k) and torch.equal(kv[:, 1], v)


def test_norm_operands_beside_each_other(env):  # noqa: F811
    torch, celty = env
    h, b = torch.randn(9, 100, device="cuda").half(), torch.randn(9, 100, device="cuda").half()
    w = torch.rand(100, device="cuda").half()
    h_out, x = torch.empty_like(h), torch.empty_like(h)
    celty.celty_block_norm(h, b, h_out, x, w_pre=w)
    one = torch.zeros(9, 4, 100, dtype=torch.float16, device="cuda")
    one[:, 0], one[:, 1] = h, b
    celty.celty_block_norm(one[:, 0], one[:, 1], one[:, 2], one[:, 3], w_pre=w)
    assert torch.equal(one[:, 0], h) and torch.equal(one[:, 1], b) and torch.equal(one[:, 2], h_out) and torch.equal(one[:, 3], x)


@pytest.mark.parametrize("which", list(WINDOWED))
def test_an_infinite_value_scale_that_is_seen(env, which):  # noqa: F811
    """What such a value stands for is not finite, and so is the result, in the
    head that reads it; it does not look like nothing seen."""
    torch, celty = env
    n, m, heads, kv_heads, window, only = WINDOWED[which]
    s = Sequences(env, [n], [m], kv_heads, 64, 32, "float16", seed=38)
    s.fill()
    q, out, ws = _attend(env, s, heads, window=window, only=only)
    at = n - m - 3   # the first tokens of the call see it, the last may not
    page, slot = int(s.table[0, at // s.page]), at % s.page
    s.cache.v_params[page, 0, slot, 0] = float("inf")
    got = torch.zeros_like(out)
    celty.celty_kv4_attention(s.cache, s.seqs, q, got, ws, window=window)
    sees = torch.arange(n - m, n, device="cuda") - window < at
    group = heads // kv_heads
    assert not got[sees][:, :group].isfinite().any()
    assert torch.equal(got[~sees], out[~sees]) and torch.equal(got[:, group:], out[:, group:])
