"""Co-run pairs that take a step as soon as they are opened, with work still
queued on the default stream and counters left by an earlier pair of the slot."""
import pytest
import torch

from paper_2606_04415_amd import flexattn as F

pytestmark = pytest.mark.gpu


def test_a_pair_steps_as_soon_as_it_is_open():
    torch.manual_seed(1)
    hq, hkv, d, P = 8, 2, 64, 16
    ns, ls = [1, 40, 1], [300, 40, 77]
    pages = [-(-n // P) for n in ls]
    bt = torch.zeros(3, max(pages), dtype=torch.int32)
    at = 0
    for s, n in enumerate(pages):
        bt[s, :n] = torch.arange(at, at + n)
        at += n
    k, v = (torch.randn(at, P, hkv, d).to(torch.bfloat16).cuda() for _ in "kv")
    q = torch.randn(sum(ns), hq, d).to(torch.bfloat16).cuda()
    qsl = [0, 1, 41, 42]
    d_qsl, d_ls, bt = (torch.tensor(x, dtype=torch.int32).cuda() for x in (qsl, ls, bt.tolist()))
    pa = F.PagedAttention(F.make_shape(hq, hkv, d, d, P, 0.125), F.make_opts(cus_decode=96, decode_tail=-1), qsl, ls, bt.shape[1])
    ref, _ = pa.alloc_out(q)
    F.flex_attn_mixed(pa.plan, pa.args(q, k, v, bt, d_ls, d_qsl, ref), F.FLEX_MODE_SERIAL)
    out, _ = pa.alloc_out(q)
    args = pa.args(q, k, v, bt, d_ls, d_qsl, out)
    a = torch.randn(4096, 4096, device="cuda", dtype=torch.bfloat16)
    b = torch.empty_like(a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for pair in range(6):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(20):                      # a few milliseconds on the default stream
            torch.matmul(a, a, out=b)
        corun = F.Corun(160, 96)
        try:
            for step in range(1 + 3 * pair):     # the counters end at a number of their own
                F.flex_attn_mixed(pa.plan, args, F.FLEX_MODE_CORUN, stream=side.cuda_stream, corun=corun)
            torch.cuda.synchronize()
        finally:
            corun.close()
        assert torch.equal(out.view(torch.int16), ref.view(torch.int16)), f"pair {pair}"
