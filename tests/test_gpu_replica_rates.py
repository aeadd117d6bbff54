"""The example that serves a replica's share of a trace: cache and attention together, graph replays among them."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_replicas_share(dtype):
    from examples import replica_rates
    r = replica_rates.run(requests=600, dtype=dtype, q_heads=8, kv_heads=2, head_dim=64, steps=5, batches=2)
    assert r["requests"] > 0 and r["new_tokens"] > 0 and r["hit_tokens"] > 0 and r["prefill_ms_per_token"] > 0 and r["decode_ms_per_token"] > 0
    # values below 6, weights that add up to 1: half a step of bf16 for the result (2^-9 of up to 6) and for the weights (the same, of the
    # sum of weights times sizes, below 6 too), twice over for the 32-bit parts
    assert r["worst"] < 2 * 2 * 6 * 2.0 ** -8
