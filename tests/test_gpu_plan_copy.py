"""A plan's copy to the device and runs on other streams than the one it is
queued on: the copy waits behind that stream's work, and the runs for the copy."""
import pytest
import torch

from paper_2606_04415_amd import flexattn as F
from paper_2606_04415_amd.workloads import WORKLOADS

from gpu_common import custom_batch, device_inputs, log, shape_of
from kv8_common import batch, bf16, cache8, scale_of, to_gpu

pytestmark = pytest.mark.gpu


def bf16_step():
    b = custom_batch(WORKLOADS["tiny"], [1, 40, 1, 3], [700, 90, 33, 3], seed=3)
    d = device_inputs(b)
    plan = lambda: F.PagedAttention(shape_of(b.workload), F.make_opts(min_split_tokens=64), b.query_start_loc, b.seq_lens,
                                    b.block_table.shape[1])

    def args(pa, out, lse):
        return pa.args(d["q"], d["k_cache"], d["v_cache"], d["block_table"], d["seq_lens"], d["query_start_loc"], out, lse)

    return d["q"], plan, args, F.flex_attn_mixed


def kv8_step():
    bt, ls, qsl, pages = batch([1, 40, 1, 3], [700, 90, 33, 3], 16, 3)
    k, v, s = to_gpu(*cache8(pages, 16, 4, 128, 3))
    q = bf16((int(qsl[-1]), 28, 128), 3).cuda()
    meta = [torch.from_numpy(x).cuda() for x in (bt, ls, qsl)]
    shape = F.make_shape(28, 4, 128, 128, 16, scale_of(128))
    plan = lambda: F.PagedAttention(shape, F.make_opts(kv_bits=8), qsl, ls, bt.shape[1])
    return q, plan, lambda pa, out, lse: pa.kv8_args(q, k, v, s, *meta, out, lse), F.flex_attn_mixed_kv8


@pytest.mark.parametrize("step", [bf16_step, kv8_step])
def test_a_run_on_another_stream_reads_the_plan_that_was_copied(step):
    q, plan, args, call = step()
    pa = plan()
    want = pa.alloc_out(q, with_lse=True)
    call(pa.plan, args(pa, *want), F.FLEX_MODE_SERIAL)
    busy = torch.randn(8192, 8192, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    outs = [pa.alloc_out(q, with_lse=True) for _ in range(3)]
    torch.cuda.synchronize()
    log(f"{step.__name__}: runs on other streams behind a late copy")
    for given, (out, lse) in zip((True, False, True), outs):
        for _ in range(20):
            busy @ busy                            # on the default stream: the copy waits for these
        p2 = plan()
        a = args(p2, out, lse)
        if given:
            call(p2.plan, a, F.FLEX_MODE_SERIAL, stream=side.cuda_stream)
        else:
            with torch.cuda.stream(side):
                call(p2.plan, a, F.FLEX_MODE_SERIAL)
        side.synchronize()
        assert torch.equal(out.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])
        torch.cuda.synchronize()


@pytest.mark.parametrize("step", [bf16_step, kv8_step])
def test_a_capture_on_another_stream(step):
    """The copy is over when a capture begins; the capture itself waits for nothing outside."""
    q, plan, args, call = step()
    pa = plan()
    want, out = pa.alloc_out(q, with_lse=True), pa.alloc_out(q, with_lse=True)
    call(pa.plan, args(pa, *want), F.FLEX_MODE_SERIAL)
    p2 = plan()
    a = args(p2, *out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(p2.plan, a, F.FLEX_MODE_SERIAL)
    for k in range(3):
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(out[1], want[1]), f"replay {k}"
    with torch.cuda.stream(torch.cuda.Stream()):   # and outside of one
        call(p2.plan, a, F.FLEX_MODE_SERIAL)
    torch.cuda.synchronize()
    assert torch.equal(out[1], want[1])
