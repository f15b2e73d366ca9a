"""What the 8-bit cache's calls refuse for its size, in every entry point that would launch it and before anything is launched (no GPU)."""
import pytest

import paper_2402_18789_amd.binding as B
from paper_2402_18789_amd import kv8
from paper_2402_18789_amd.host import c_cfg
from test_kv8_host import R, full_library, host_maps, refused
from workload import CONFIGS


@full_library
@pytest.mark.parametrize("reqs", [[R(0, 0, 5, 1), R(1, 1, 0, 30)], [R(0, 0, 5, 1), R(0, 1, 3, 1)]], ids=["mixed", "single tokens"])
@pytest.mark.parametrize("heads,head_dim", [(174, 256), (1533, 16)])
def test_more_kv_heads_than_a_token_s_block_holds(reqs, heads, head_dim):
    """(every address is a number: nothing is read or written)"""
    cfg = CONFIGS["c1_tiny_f32"].with_(n_q_heads=heads, n_kv_heads=heads, head_dim=head_dim, lora_targets=())
    c = c_cfg(cfg)
    m, keep = host_maps(reqs, {0: [3], 1: [2, 0]}, 16, 8, heads, heads)
    n_runs = len(kv8.flexco_kv8_runs(m))
    pool = kv8.Pool(4096, 8192, 64, 128, 8, 16)
    big, w = 1 << 40, B.BaseWeights(16, None, *[16 * i for i in range(2, 7)])
    assert str(heads) in refused(B.FLEXCO_EUNSUPPORTED, kv8.flexco_kv8_append, c, m, 256, n_runs, big, pool, 2 * big, cfg.q_dim, 0)
    assert str(heads) in refused(B.FLEXCO_EUNSUPPORTED, kv8.flexco_kv8_layer_forward, c, w, None, m, 256, n_runs, big, 2 * big, pool, None, 64, big, 0)
