"""Sizes of the chunk attention's workspace, which belong to one call each."""
import pytest
import torch

jfkv = pytest.importorskip("paper_2609_17475_amd.jfkv")
LAY = jfkv.layout(256, 8, 128, 64, 300)


def need(T, prefix):
    return jfkv.jf_kv8_prefill_workspace_bytes(LAY, T, 32, prefix)


def test_shorter_calls_can_need_more():
    assert need(64, 30000) > need(64, 65536) > 0
    assert need(1024, 1000) > need(2048, 65536) == 0


@pytest.mark.gpu
def test_one_workspace_serves_a_prompt_in_chunks():
    """Chunks of 512 rows and a partial last one: the largest of the sizes does, and
    NULL where the last chunk needs more than the others left it."""
    import numpy as np
    from oracle import kv8 as ref
    from tests.kv8_cases import Pair, check_out, i32, rows, wide
    rng = np.random.default_rng(0)
    P, hkv, hq, d, n = 256, 2, 4, 128, 1100
    p = Pair(P, hkv, d, 64, 6)
    table = np.array([3, 1, 5, 0, 4], np.int32)
    p.fill(rng, [n], table[None])
    q = rows(rng, n, hq, d, False, 0.7)
    spans = [(0, 512), (512, 1024), (1024, 1100)]
    sizes = [jfkv.jf_kv8_prefill_workspace_bytes(p.lay, b - a, hq, a) for a, b in spans]
    ws = torch.full((max(sizes),), 0xFF, dtype=torch.uint8, device="cuda")
    short = ws[:max(sizes) // 32 * 16]
    r = ref.attend(p.host, wide(q), table, n, 0.1)
    out = torch.empty_like(q, device="cuda")
    for space in (ws, short):
        out.fill_(float("nan"))
        for (a, b), size in zip(spans, sizes):
            call = (p.gpu, q[a:b].cuda(), i32(table), a, 0.1, out[a:b])
            if size > space.numel():
                with pytest.raises(jfkv.JfError):
                    jfkv.jf_kv8_prefill_attn(*call, workspace=space)
            jfkv.jf_kv8_prefill_attn(*call, workspace=space if size <= space.numel() else None)
        check_out(out, r, d, False)
