"""The example that runs the four-bit operators with the prompt's (examples/decode_four_bits.py) on a small layer: a decoded token is what the
prompt gives for the same token, whether the cache stayed on the device or went to the host and back, in a graph or not."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode_four_bits", os.path.join(ROOT, "examples", "decode_four_bits.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _near(got, want):
    # the project's bar for bf16 results that went different ways: 2e-2 of the largest value
    assert torch.isfinite(got).all() and (got - want).abs().max().float() <= 2e-2 * want.abs().max().float(), float((got - want).abs().max() / want.abs().max())


@pytest.mark.parametrize("heads,kv_heads,d,page", [(4, 2, 64, 16), (7, 1, 128, 64), (2, 2, 256, 32)])
def test_a_decoded_token_is_the_prompts(example, heads, kv_heads, d, page):
    S, H, I = 200, 256, 512
    x = torch.randn((S + 3, H), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(torch.bfloat16)
    whole = example.Layer(H, I, heads, kv_heads, d, S + 3, page)
    want = whole.prompt(x, chunk=77, mini_seq=50)                # chunks end inside pages
    layer = example.Layer(H, I, heads, kv_heads, d, S + 3, page)
    host, side = torch.empty(layer.cache.numel(), dtype=torch.uint8, pin_memory=True), torch.cuda.Stream()
    layer.prompt(x[:S], chunk=page * 3, mini_seq=64, offload=(host, side))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    kept = layer.cache.clone()
    layer.cache.fill_(255)
    layer.restore(host, torch.cuda.current_stream())
    torch.cuda.synchronize()
    used = -(-S // page)
    assert torch.equal(layer.cache[:used], kept[:used])
    step_in = x[S:S + 1].clone()
    layer.set_place(S)
    _near(layer.token(step_in), want[S:S + 1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_out = layer.token(step_in)
    for i in (S, S + 1, S + 2):
        layer.set_place(i)
        step_in.copy_(x[i:i + 1])
        graph.replay()
        replayed = step_out.clone()
        eager = layer.token(x[i:i + 1].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(replayed.view(torch.int16), eager.view(torch.int16))
        _near(eager, want[i:i + 1])
