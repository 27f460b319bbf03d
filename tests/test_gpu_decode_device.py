"""The operators around the products launch on the current GPU: their binding
refuses tensors and streams of another.  One GPU is enough to see it: which one is
current, and which one a stream is on, are made up."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls():
    import torch
    import paper_2608_01536_amd as celty
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    z = dict(dtype=torch.float16, device="cuda")
    h, x = torch.ones(2, 64, **z), torch.empty(2, 64, **z)
    cache = celty.Kv4Cache(1, 2, 64, 32)
    seqs = celty.Kv4Seqs(torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    k, q, out = torch.ones(1, 2, 64, **z), torch.ones(1, 4, 64, **z), torch.empty(1, 4, 64, **z)
    ws = celty.new_kv4_workspace(cache, seqs, 1, 4)
    tokens, ws2 = torch.empty(2, dtype=torch.int32, device="cuda"), celty.new_sample_workspace(h)
    return torch, [lambda **s: celty.celty_block_norm(h, None, None, x, **s), lambda **s: celty.celty_kv4_append(cache, seqs, k, k, **s),
                   lambda **s: celty.celty_kv4_gather(cache, seqs, k, k.clone(), **s),
                   lambda **s: celty.celty_kv4_attention(cache, seqs, q, out, ws, **s),
                   lambda **s: celty.celty_sample(h, None, tokens, ws2, **s)]


def test_another_current_device_is_refused(calls, monkeypatch):
    torch, calls = calls
    stream = torch.cuda.current_stream()
    for call in calls:
        call()
        call(stream=stream)
        call(stream=int(stream.cuda_stream))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in calls:
        for s in (dict(), dict(stream=stream), dict(stream=int(stream.cuda_stream))):
            with pytest.raises(ValueError, match="current device"):
                call(**s)


def test_a_stream_of_another_device_is_refused(calls):
    torch, calls = calls

    class Elsewhere:
        device = torch.device("cuda", 1)
        cuda_stream = torch.cuda.current_stream().cuda_stream
    for call in calls:
        with pytest.raises(ValueError, match="stream"):
            call(stream=Elsewhere())
