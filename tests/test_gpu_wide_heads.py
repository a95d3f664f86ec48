"""Decode with more than eight KV heads that eight does not divide: the last
column of work-groups covers fewer heads than the others, and the merge of
split sequences writes the rows of those heads only. Every output and
log-sum-exp against the oracle, and the rows behind the last sequence's, which
belong to no token, as they were."""
import numpy as np
import pytest
import torch

import oracle.attention as OA
from paper_2606_04415_amd import flexattn as F
from paper_2606_04415_amd.workloads import WORKLOADS

from gpu_common import check_close, custom_batch, device_inputs, log, shape_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv", [(20, 20), (24, 12), (45, 9)])
def test_split_decode_writes_its_own_rows(hq, hkv):
    b = custom_batch(WORKLOADS["decode"], [1, 1, 1], [700, 30, 900], seed=5, num_q_heads=hq, num_kv_heads=hkv)
    w, d = b.workload, device_inputs(b)
    pa = F.PagedAttention(shape_of(w), F.make_opts(min_split_tokens=64), b.query_start_loc.tolist(), b.seq_lens.tolist(),
                          b.block_table.shape[1])
    assert pa.plan.info["n_split_seqs"] >= 2 and pa.plan.info["decode_wg_width"] > 1
    log(f"split decode, {hq}/{hkv} heads in columns of 8 KV heads")
    out = torch.full((3 + 8, hq, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((3 + 8, hq), 5.0, dtype=torch.float32, device="cuda")
    args = pa.args(d["q"], d["k_cache"], d["v_cache"], d["block_table"], d["seq_lens"], d["query_start_loc"], out[:3], lse[:3])
    F.flex_attn_decode(pa.plan, args)
    torch.cuda.synchronize()
    ref_o, ref_l = OA.paged_attention(b.q, b.k_cache, b.v_cache, b.block_table, b.seq_lens, b.query_start_loc, w.sm_scale,
                                      num_kv_heads=hkv, page_size=w.page_size)
    check_close(out[:3].cpu(), ref_o, f"{hq}/{hkv} out")
    check_close(lse[:3].cpu(), ref_l, f"{hq}/{hkv} lse")
    assert (out[3:] == 5.0).all() and (lse[3:] == 5.0).all(), "rows behind the last token changed"
