"""Which operands of the operators around the products may lie beside each other:
rows of one larger tensor that share no element are accepted, rows that do are
refused.  The rule, for every combination of strides, against a set of addresses."""
import ctypes
import itertools

import pytest

from paper_2608_01536_amd import CELTY_EINVAL, decode
from tests.test_abi import host_only
from tests.test_decode_abi import F16, F32, FAKE, _cache, _norm_call, _seqs

B = ctypes.byref
WS = FAKE + 0x10000000


def _attention(q, out, n_tokens, heads):
    """Status of a call on fake addresses: without a GPU, what passes the checks ends
    in the launch's own error."""
    c, s = _cache(head_dim=64, kv_heads=1), _seqs(n_tokens=n_tokens)
    return decode._attention(B(c), B(s), F16, heads, B(decode.celty_heads(*q)), B(decode.celty_heads(*out)), 0.1, 0, WS, 1 << 40, None)


def _gather(k, v, n_tokens, heads):
    c, s = _cache(head_dim=64, kv_heads=heads), _seqs(n_tokens=n_tokens)
    return decode._gather(B(c), B(s), F16, B(decode.celty_heads(*k)), B(decode.celty_heads(*v)), None)


def _elements(t, n, heads, D=64):
    """Start elements, in units of 8, of every 8 channels that a tensor holds; None where it holds one twice."""
    data, ts, hs = t
    e = [(data - FAKE) // 2 + i * ts + h * hs + d for i in range(n) for h in range(heads) for d in range(0, D, 8)]
    return set(e) if len(set(e)) == len(e) else None


def _tensors(n, heads):
    strides = [64, 128, 192, 64 * heads, 128 * heads, 64 * n, 128 * n, 64 * n * heads, 320]
    for ts, hs in itertools.product(strides, strides):
        yield ts, hs


@host_only
@pytest.mark.parametrize("n,heads", [(2, 2), (5, 4), (3, 1), (4, 3)])
def test_outputs_whose_rows_meet_are_refused(n, heads):
    far = FAKE + 0x8000000
    seen = set()
    for ts, hs in _tensors(n, heads):
        t = (FAKE, ts, hs)
        ok = _elements(t, n, heads) is not None
        seen.add(ok)
        assert (_attention((far, 64 * heads, 64), t, n, heads) != CELTY_EINVAL) == ok, t
        assert (_gather((far, 64 * heads, 64), t, n, heads) != CELTY_EINVAL) == ok, t
        assert (_gather(t, (far, 64 * heads, 64), n, heads) != CELTY_EINVAL) == ok, t
    assert seen == {True, False} or heads == 1


@host_only
@pytest.mark.parametrize("n,heads", [(2, 2), (5, 4), (3, 1), (4, 3)])
def test_tensors_of_one_buffer(n, heads):
    """The same strides, one tensor a little behind the other."""
    for ts, hs in _tensors(n, heads):
        a = _elements((FAKE, ts, hs), n, heads)
        if a is None:
            continue
        for offset in (8, 56, 64, 72, 128, 64 * heads, 64 * heads - 8, 64 * n, 192, 320, 1024, 4096):
            for one, two in (((FAKE, ts, hs), (FAKE + 2 * offset, ts, hs)), ((FAKE + 2 * offset, ts, hs), (FAKE, ts, hs))):
                ok = not (_elements(one, n, heads) & _elements(two, n, heads))
                # starts are whole multiples of 8 elements, so rows meet in whole pieces
                assert (_attention(one, two, n, heads) != CELTY_EINVAL) == ok, (one, two)
                assert (_gather(one, two, n, heads) != CELTY_EINVAL) == ok, (one, two)


@host_only
def test_gather_into_one_tensor_twice_is_refused():
    t = (FAKE, 128, 64)
    assert _gather(t, t, 3, 2) == CELTY_EINVAL
    assert _gather(t, (FAKE + 2 * 3 * 128, 128, 64), 3, 2) != CELTY_EINVAL


@host_only
@pytest.mark.parametrize("res", [F16, F32])
def test_norm_of_columns_of_one_buffer(res):
    """h, b, h_out, x and gate as columns of one matrix of bytes."""
    rs = 4 if res == F32 else 2
    n, rows, far = 64, 4, 0x800000
    ld = 1024   # bytes
    wh, wx = n * rs, n * 2

    def call(h, b, out, x, gate=None, ld_gate=0):
        return _norm_call(rows=rows, n=n, res=res, h=FAKE + h, ldh=ld // rs, b=FAKE + b, ldb=ld // 2, out=FAKE + out, ldo=ld // rs,
                          x=FAKE + x, ldx=ld // 2, gate=None if gate is None else FAKE + gate, ld_gate=ld_gate) != CELTY_EINVAL
    assert call(0, wh, wh + wx, 2 * wh + wx)                       # four neighbours
    assert call(0, wh, 0, wh)                                      # both in place
    assert call(512, wh, 512, 0)                                   # x before h
    assert call(0, wh, wh + wx, 2 * wh + wx, 2 * wh + 2 * wx, ld // 2)
    assert call(0, wh, wh + wx, 2 * wh + wx, 2 * wh + 2 * wx, 0)   # one gate beside the first row's x
    for ld_gate in (ld // 2, 0):                                   # the gate's first element is x's last
        assert not call(0, wh, wh + wx, 2 * wh + wx, 2 * wh + 2 * wx - 2, ld_gate)
    assert not call(0, wh, wh + wx - rs, 2 * wh + wx)              # h_out begins in b
    assert not call(0, wh, rs, far)                                # h_out is h, moved by an element
    assert not call(0, wh, ld, far)                                # by a row: read after it is written
    assert call(0, wh, rows * ld, far)                             # by all rows
    assert not call(0, wh, far, far + wh - 2)                      # x begins in h_out
    assert call(0, wh, far, far + wh) and call(0, wh, far + wx, far)
    assert not call(0, wh, far, far + ld - 2)                      # x ends in the next row's h_out
    assert call(0, wh, far, far + ld - wx)


@host_only
def test_a_stride_along_one_element_is_of_no_matter():
    odd = 12345
    for n, heads, a, b in ((1, 4, (FAKE, odd, 64), (FAKE + 0x100000, -odd, 64)), (3, 1, (FAKE, 64, odd), (FAKE + 0x100000, 64, 0)),
                           (1, 1, (FAKE, 1 << 40, -3), (FAKE + 0x100000, 5, 1 << 50))):
        seqs = _seqs(n_tokens=n)
        c = _cache(head_dim=64, kv_heads=heads)
        x, y = decode.celty_heads(*a), decode.celty_heads(*b)
        for f in (decode._append, decode._gather):
            assert f(B(c), B(seqs), F16, B(x), B(y), None) != CELTY_EINVAL, (n, heads)
        assert decode._attention(B(c), B(seqs), F16, heads, B(x), B(y), 0.1, 0, WS, 1 << 40, None) != CELTY_EINVAL, (n, heads)
