"""celty_sample on rows that the choice of a token must not be sensitive to:
logits with an offset, filters at the ends of their ranges.  The definition is
that of tests/test_gpu_sample.py."""
import pytest

from tests.test_gpu_sample import _rows, _sample, _want, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("p", [float("-inf"), -3.0e38, -1.0, -0.0, 0.0, 1e-45])
def test_top_p_that_keeps_the_first_token_alone(env, p):  # noqa: F811
    """Also beside a top-k whose bin is the largest logit's."""
    torch, _ = env
    for dtype in ("float16", "float32"):
        logits, noise = _rows(torch, 6, 5003, dtype, 41)
        flat, _ = _rows(torch, 6, 5003, dtype, 42, sharp=False)
        for x in (logits, flat, torch.zeros_like(logits)):
            for f in (dict(p=p), dict(p=p, k=1), dict(p=p, k=7), dict(p=p, k=3000), dict(p=p, k=9000), dict(p=p, m=0.2, k=50)):
                got = _sample(env, x, noise, **f)
                assert (got == x.float().cpu().numpy().argmax(1)).all(), (dtype, f)
                assert (got == _want(x, noise, **f)).all()


def _offset_rows(torch, rows, V, offset, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    logits = (offset + 2 * torch.randn(rows, V, generator=g, device="cuda")).to(dtype)
    return logits, torch.empty(rows, V, device="cuda").exponential_(generator=g)


OFFSETS = [0.0, 8.0, 20.0, -20.0, -40.0, 300.0, -1000.0]


@pytest.mark.parametrize("offset", OFFSETS)
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_logits_with_an_offset(env, offset, dtype):  # noqa: F811
    """The token depends on differences of logits only; so does how it is found."""
    torch, _ = env
    for V in (5001, 32000, 100277):
        logits, noise = _offset_rows(torch, 2, V, offset, getattr(torch, dtype), V)
        for f in (dict(p=0.9), dict(p=0.5, T=1.7), dict(k=400, p=0.9), dict(k=3000), dict(k=3000, p=0.97, T=0.4), dict(p=0.99, m=1e-4)):
            assert (_sample(env, logits, noise, **f) == _want(logits, noise, **f)).all(), (V, f)


@pytest.mark.parametrize("offset", OFFSETS[1:])
@pytest.mark.parametrize("V", [32000, 100277])
def test_an_offset_does_not_change_the_time(env, offset, V):  # noqa: F811
    """Rows without runs of equal logits are cut from a list of a few thousand
    tokens at most, wherever they lie; one workgroup alone takes 20 times as long."""
    torch, celty = env
    p = torch.full((2,), 0.9, device="cuda")
    tokens = torch.empty(2, dtype=torch.int32, device="cuda")

    def best_time(at):
        logits, noise = _offset_rows(torch, 2, V, at, torch.float32, 43)
        ws = celty.new_sample_workspace(logits)
        times = []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                celty.celty_sample(logits, noise, tokens, ws, top_p=p)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    plain = best_time(0.0)
    assert best_time(offset) < 4 * plain


@pytest.mark.parametrize("dtype,offset", [("bfloat16", 8.0), ("bfloat16", 20.0), ("bfloat16", -20.0), ("float16", -40.0), ("float16", 100.0)])
def test_equal_logits_in_thousands_do_not_change_the_time(env, dtype, offset):  # noqa: F811
    """16-bit logits with an offset are runs of equal ones, up to two thousand here."""
    torch, celty = env
    V = 100277
    p = torch.full((2,), 0.9, device="cuda")
    tokens = torch.empty(2, dtype=torch.int32, device="cuda")

    def best_time(at):
        logits, noise = _offset_rows(torch, 2, V, at, getattr(torch, dtype), 44)
        ws = celty.new_sample_workspace(logits)
        times = []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                celty.celty_sample(logits, noise, tokens, ws, top_p=p)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    plain = best_time(0.0)
    assert best_time(offset) < 3 * plain


@pytest.mark.parametrize("run", [65, 300, 1025, 2000, 4096, 4097, 9000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_cuts_within_runs_of_equal_logits(env, run, dtype):  # noqa: F811
    """Runs below a few larger logits, spread over the row or side by side, one
    near another: the lower indices are kept."""
    torch, _ = env
    V = 20011
    g = torch.Generator(device="cuda")
    g.manual_seed(run)
    x = torch.full((6, V), -30.0, device="cuda")
    for r in range(6):
        at = torch.randperm(V, generator=g, device="cuda")[:run] if r % 2 else torch.arange(700, 700 + run, device="cuda")
        x[r, at] = 3.0
        more = torch.randperm(V, generator=g, device="cuda")[:30]
        x[r, more[:20]] = 3.0 + 0.25 * torch.arange(20, device="cuda") / (1 + r)
        x[r, more[20:]] = 2.984375
    x = x.to(getattr(torch, dtype))
    noise = torch.empty(6, V, device="cuda").exponential_(generator=g)
    one = torch.ones_like(noise)
    one[:, ::7] = 0.5
    for f in (dict(k=21), dict(k=run // 2), dict(k=run + 9), dict(k=run + 25), dict(p=0.3), dict(p=0.9), dict(k=run - 1, p=0.7), dict(k=40, p=0.999)):
        for e in (noise, one):
            assert (_sample(env, x, e, **f) == _want(x, e, **f)).all(), f
