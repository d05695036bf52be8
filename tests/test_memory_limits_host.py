"""Host-side checks (no kernel launches) of the sizes that attention over an 8-bit cache and linear attention take, and of the workspaces that they ask for."""
import pytest

import paper_2604_12841_amd as pdx
from paper_2604_12841_amd import tokens
from test_memory_host import CACHE, LONG, attention8, linear

BIG = 2147483647


@pytest.mark.parametrize("kw", [dict(batch=65535, kv_heads=200, heads=200), dict(batch=65535, kv_heads=128, heads=8192), dict(batch=32768, kv_heads=256, heads=256),
                                dict(batch=65535, kv_heads=65535, heads=65535)])
def test_launches_stay_below_2_32_threads(kw):
    """512 threads for each 16 rows of a key head, 256 for each 128 where there are more than 64."""
    size = dict(head_dim=16, capacity=1, n_q=1, q_head_stride=16, out_head_stride=16, q_batch_stride=1 << 24, out_batch_stride=1 << 24)
    assert attention8(**(size | kw)) == pdx.PD_ERR_UNSUPPORTED


def work8(**kw):
    return tokens._functions().predecoder_attention8_workspace(tokens.Attention8Args(**(CACHE | dict(heads=4, scale=0.1, n_q=1) | kw)))


def work_linear(**kw):
    return tokens._functions().predecoder_linear_attention_workspace(tokens.LinearAttentionArgs(**(LONG | kw)))


def test_workspaces_at_the_end_of_the_sizes():
    """What is refused asks for nothing; attention for a GB of results at most and 8 bytes for each row of them; linear attention for a state a workgroup."""
    for kw in (dict(capacity=BIG), dict(capacity=BIG, head_dim=16), dict(capacity=BIG, head_dim=128, n_q=1000), dict(batch=60, kv_heads=1, heads=1, capacity=BIG, n_q=16)):
        assert 0 < work8(**kw) <= (1 << 30) + (1 << 26)
    for kw in (dict(capacity=BIG, n_q=1 << 24), dict(batch=65535, n_q=64, capacity=BIG), dict(capacity=0), dict(capacity=1), dict(capacity=BIG, n_q=BIG),
               dict(capacity=BIG, heads=130), dict(capacity=BIG, head_dim=24), dict(capacity=BIG, batch=65535, kv_heads=256, heads=256)):
        assert work8(**kw) == 0
    for kw in (dict(n=BIG // 2, per_round=1), dict(n=BIG // 2, per_round=40), dict(head_dim=128, n=1 << 28), dict(head_dim=8, n=1 << 28), dict(n=5000, heads=64, kv_heads=2)):
        assert 0 < work_linear(**kw) <= 16 << 20
    for kw in (dict(n=BIG // 2, per_round=BIG), dict(n=1, per_round=BIG), dict(n=0), dict(batch=65535), dict(n=BIG), dict(n=1 << 29, heads=4), dict(batch=BIG, n=1),
               dict(head_dim=12), dict(per_round=0), dict(n=1 << 28, batch=4000)):
        assert work_linear(**kw) == 0


@pytest.mark.parametrize("kw", [dict(batch=BIG, n=1), dict(batch=1 << 23, n=1), dict(batch=1 << 23, n=2), dict(batch=BIG, heads=BIG, kv_heads=BIG, n=1),
                                dict(batch=1 << 22, n=3, head_dim=128), dict(batch=BIG, heads=BIG, kv_heads=BIG, n=0)])
def test_linear_launches_stay_below_2_32_threads(kw):
    """256 threads for each key head of an entry, of more than 64 channels and several tokens twice as many."""
    size = {n + "_batch_stride": 1 << 20 for n in ("q", "k", "v", "out")}
    assert linear(**(size | dict(heads=2, kv_heads=2) | kw)) == pdx.PD_ERR_UNSUPPORTED
