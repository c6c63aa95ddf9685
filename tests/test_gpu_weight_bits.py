"""sfi_weight_attn: the softmax weights go into the outputs with all of their bits."""
import pytest

from cache_ref import i32
from test_gpu_shared_edges import EXACT, _two_terms_miss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("B, Hq, Hkv, n", [(1, 8, 2, 512), (3, 16, 1, 700), (32, 32, 8, 1024)])
def test_weights_keep_their_bits(B, Hq, Hkv, n, page):
    """Half of the rows with a weight of 1 and values of 0, half with a weight that two bf16 terms miss by 2^-18 or more and values of 1 (the bound: where EXACT is)."""
    import torch
    import paper_2603_12038_amd as sfi

    xs = _two_terms_miss()
    K, V = torch.zeros((n, 128), dtype=torch.bfloat16), torch.zeros((n, 128), dtype=torch.bfloat16)
    K[1::2, 0], V[1::2] = 1.0, 1.0
    if page:
        pages = (n + page - 1) // page
        pools = [torch.zeros((pages * page, 128), dtype=torch.bfloat16) for _ in range(2)]
        pools[0][:n], pools[1][:n] = K, V
        K, V = (t.view(pages, 1, page, 128).cuda().expand(pages, Hkv, page, 128) for t in pools)  # strides of zero: all heads hold the same rows
    else:
        K, V = (t.cuda().expand(B, Hkv, n, 128) for t in (K, V))
    ctx = sfi.SfiContext(B, Hq, Hkv, n, 64, 4, 64, K, V, page_size=page, page_layout="htd")
    try:
        if page:
            table = torch.arange(pages, dtype=torch.int32).repeat(B, 1).cuda()
            sfi.sfi_set_block_table(ctx.handle, table, pages)
        x = xs[torch.arange(B * Hq) * 7919 % len(xs)].view(B, Hq)
        q = torch.zeros((B, Hq, 128), dtype=torch.bfloat16)
        q[:, :, 0] = -x.to(torch.bfloat16)
        q, out, w = q.cuda(), torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hkv, n), device="cuda")
        print(f"[gpu-weight-bits] B={B} heads {Hq}/{Hkv} rows {n} page {page}", flush=True)
        sfi.sfi_weight_attn(ctx.handle, q, K, V, i32([n] * B), 0, 1.0, None, w, out)
        torch.cuda.synchronize()
        p = torch.exp(-x / 128.0 ** 0.5)
        odd = n // 2
        want = (odd * p / (n - odd + odd * p))[:, :, None]
        off = out.cpu().double() / want - 1
        assert off.square().mean().sqrt().item() <= EXACT
    finally:
        ctx.close()
