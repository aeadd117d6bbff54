"""Kernels over the cache keep everything in registers: what the built library says of their scratch memory."""
from paper_2602_11688_amd import build


def test_attention_and_appends():
    kernels = {}
    for elf in build._code_objects(build.LIB):
        kernels.update(build._kernels(elf))
    found = {name: scratch for name, (_, scratch) in kernels.items() if any(part in name for part in ("attend_", "join_prompt", "append_kernel", "kv_"))}
    assert len(found) > 100
    assert {name: scratch for name, scratch in found.items() if scratch} == {}
