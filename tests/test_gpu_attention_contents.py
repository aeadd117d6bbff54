"""Workspaces, offsets and lengths of any content in the attention over the paged cache and in the cache itself."""
import pytest

import paper_2602_11688_amd as g
from tests.attention_helpers import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type,d,page", [("bf16", 128, 64), ("e4m3", 64, 48)])
def test_a_workspace_of_a_large_batch_serves_every_smaller_one(type, d, page):
    """Sized once, for many tokens of many sequences that need no pieces, and then used for few, which do, and for single tokens."""
    large = Case([(3000, 9000)] * 4, q_heads=4, kv_heads=1, d=d, page=page, type=type, columns=20000 // page + 1)
    ws = g.attend_workspace(large.cache, large.batch, 4)
    check(large, g.attend_prompt(large.cache, large.batch, large.q, lse=True, workspace=ws))
    for spec, token in (([(3, 20000)], False), ([(1, 20000), (1, 3), (1, 777)], True), ([(500, 7000), (1, 9)], False), ([(1, 20000)], True)):
        c = Case(spec, q_heads=4, kv_heads=1, d=d, page=page, type=type, token=token)
        check(c, (g.attend_token if token else g.attend_prompt)(c.cache, c.batch, c.q, lse=True, workspace=ws))
