"""The limits of an attention call's workgroups, at their values (no GPU: the
workspace of a call that would be refused is 0)."""
import pytest

from paper_2407_17353_amd import binding as sc

AT = 0x10000000  # (a device array's address, never read here)


def opts(**kw):
    o = dict(heads=1, kv_heads=1, head_dim=16, causal=1, batch=1, softmax_scale=0.25, q_start=AT, k_start=AT, k_len=None, max_q=0,
             max_k=0)
    o.update(kw)
    return sc.CAttentionOpts(*o.values())


@pytest.mark.parametrize("kw,rows_q,rows_k,good", [
    (dict(batch=2048, heads=32, kv_heads=32), 32768, 32768, True),       # past 2^24 workgroups
    (dict(batch=1 << 21, max_k=128), 32768, 32768, False),               # 2^31 of 32 query columns
    (dict(batch=1 << 21, max_k=128, max_q=32736), 32768, 32768, True),
    (dict(batch=(1 << 21) - 1, max_k=128), 32768, 32768, True),
    (dict(batch=1 << 20, max_k=128, heads=2), 32768, 32768, False),
    (dict(batch=1 << 23, max_q=32), 32768, 32768, False),                # 2^31 of 128 keys
    (dict(batch=1 << 23, max_q=32, max_k=32640), 32768, 32768, True),
    (dict(batch=1 << 15, heads=65536, kv_heads=65536, max_q=1, max_k=1), 64, 64, False),
    (dict(batch=(1 << 15) - 1, heads=65536, kv_heads=65536, max_q=1, max_k=1), 64, 64, True),
    (dict(batch=1 << 30, heads=65536, kv_heads=65536), 1 << 20, 1 << 30, False),
    (dict(heads=16), 1 << 26, 1, True),                                  # 2^30 queries times heads of a key head
    (dict(heads=16), (1 << 26) + 1, 1, False),
])
def test_workgroups(kw, rows_q, rows_k, good):
    n = sc.scalify_attention_bwd_workspace_size(rows_q, rows_k, opts(**kw), sc.RESCALE_NONE)
    assert (n > 0) == good
