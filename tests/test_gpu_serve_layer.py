"""The serving operators together, as examples/serve_layer.py uses them, against the same layer in FP32.

Tolerance.  A block's largest of 32 normal values is about 2.2 sigma and lies between 3.5 and 7 steps of its 4-bit mantissas, so a stored
value is off by a uniform error of a step, 0.09 to 0.18 sigma.  Values carry it to the output whole (0.18 at most); keys carry it to
the scores, which are of order one, and so to the weights (another 0.18, relative); 8-bit codes add some 0.01 each.  Together at
most 0.26; 0.3 leaves room for the spread of few conversations.  A step that sees one token too many, or the wrong slot, is off by 1."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("conversations,steps,heads,kv_heads,dim,prompt,evictions", [
    (8, 96, 8, 2, 64, 200, 1),
    (3, 40, 4, 4, 80, 30, 0),
    (1, 400, 8, 1, 128, 255, 3),
])
def test_layer_follows_the_fp32_layer(conversations, steps, heads, kv_heads, dim, prompt, evictions):
    from examples.serve_layer import run
    print(f"[layer] {conversations} conversations, {heads}/{kv_heads} heads of {dim}, prompt {prompt}, {steps} steps", flush=True)
    error, times = run(conversations, steps, heads, kv_heads, dim, prompt=prompt)
    assert times == evictions
    assert error < 0.3
