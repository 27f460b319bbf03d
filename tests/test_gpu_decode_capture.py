"""Capturing the step of examples/decode_step.py leaves it at its start."""
import pytest

from tests.test_gpu_decode_step import example  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [0, 7, 16])
def test_capture_leaves_a_state_as_after_reset(example, steps):  # noqa: F811
    """After no steps, some, and all that the cache has room for."""
    torch, mod = example
    dec = mod.Decoder(mod.Config(layers=1, vocabulary=1001, ffn=500, max_tokens=16, page_tokens=32), seed=2)
    dec.reset(9)
    for _ in range(steps):
        dec.step()
    token = int(dec.token[0])
    graph = dec.capture()
    assert int(dec.kv_len[0]) == 0 and int(dec.token[0]) == token
    graph.replay()
    torch.cuda.synchronize()
    first = dec.logits.clone()
    assert int(dec.kv_len[0]) == 1
    dec.reset(token)
    dec.step()
    assert torch.equal(dec.logits, first)
