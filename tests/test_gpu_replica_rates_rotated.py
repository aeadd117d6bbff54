"""The example that serves a replica's share of a trace, with heads normed and rotated and attention over a window and first tokens."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,window,sinks", [("bf16", 700, 4), ("e4m3", 0, 0), ("e4m3", 300, 130)])
def test_a_replicas_share_rotated(dtype, window, sinks):
    from examples import replica_rates
    r = replica_rates.run(requests=600, dtype=dtype, q_heads=8, kv_heads=2, head_dim=64, steps=5, batches=2, rotate=True, window=window, sinks=sinks)
    assert r["requests"] > 0 and r["new_tokens"] > 0 and r["hit_tokens"] > 0 and r["prefill_ms_per_token"] > 0 and r["decode_ms_per_token"] > 0
    # values below 6, weights that add up to 1: half a step of bf16 for the result (2^-9 of up to 6) and for the weights (the same, of the
    # sum of weights times sizes, below 6 too), twice over for the 32-bit parts
    assert r["worst"] < 2 * 2 * 6 * 2.0 ** -8
