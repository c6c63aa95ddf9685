"""sfi_rope_append for a batch with unused slots, and queries that are written where they are read."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["head", "thd"])
@pytest.mark.parametrize("new", [1, 5])
def test_unused_slots_take_no_rows_and_raise_no_flag(layout, new):
    """ctx_len 0 with every sequence getting `new` rows: nothing is written for the slot, and nothing is reported."""
    import torch
    import paper_2603_12038_amd as sfi

    lens = [20, 0, new, 0]
    cache = ref.Cache(4, 2, 32, layout, seed=15)
    ctx = cache.context(4)
    try:
        sfi.sfi_set_rope(ctx.handle, 64)
        before = [cache.numpy(0), cache.numpy(1)]
        g = torch.Generator().manual_seed(16)
        q, k = (torch.randn((4, new, h, 128), generator=g).to(torch.bfloat16).cuda() for h in (4, 2))
        q_out = torch.full_like(q, 7.0)
        sfi.sfi_rope_append(ctx.handle, q, k, k, i32(lens), None, None, q_out, cache.K, cache.V)
        torch.cuda.synchronize()
        assert sfi.sfi_device_status(ctx.handle) == 0
        after = [cache.numpy(0), cache.numpy(1)]
        for b, n in enumerate(lens):
            if n == 0:
                assert (bits(q_out)[b] == bits(torch.tensor([7.0], dtype=torch.bfloat16))[0]).all()
                assert all(np.array_equal(x[b], y[b]) for x, y in zip(after, before))
            else:
                assert np.array_equal(after[1][b, :, n - new:n].transpose(1, 0, 2), bits(k)[b])
        # a length that is there but does not hold the new rows is still reported
        sfi.sfi_rope_append(ctx.handle, None, k, k, i32([20, 0, max(new - 1, 1), 0]), None, None, None, cache.K, cache.V)
        torch.cuda.synchronize()
        assert sfi.sfi_device_status(ctx.handle) == (sfi.binding.GUARD_N_NEW if new > 1 else 0)
    finally:
        ctx.close()


def test_a_dimension_of_one_may_have_any_stride():
    """One new row per sequence out of a tensor whose row stride is odd: the same bits as from a contiguous one."""
    import torch
    import paper_2603_12038_amd as sfi

    caches = [ref.Cache(3, 2, 32, "head", seed=17) for _ in range(2)]
    got = []
    for cache, stride in zip(caches, (512, 5)):
        ctx = cache.context(4)
        try:
            sfi.sfi_set_rope(ctx.handle, 128)
            g = torch.Generator().manual_seed(18)
            q, k = (torch.randn(3 * h * 128, generator=g).to(torch.bfloat16).cuda().as_strided((3, 1, h, 128), (h * 128, stride, 128, 1)) for h in (4, 2))
            q_out = torch.zeros((3, 1, 4, 128), dtype=torch.bfloat16, device="cuda")
            sfi.sfi_rope_append(ctx.handle, q, k, k, i32([9, 1, 32]), None, None, q_out, cache.K, cache.V)
            torch.cuda.synchronize()
            got.append([bits(q_out), cache.numpy(0), cache.numpy(1)])
        finally:
            ctx.close()
    assert all(np.array_equal(a, b) for a, b in zip(*got))


def test_queries_in_place_have_to_be_laid_out_like_the_output():
    """Refused on the host, before anything is launched: q_out at q, whose rows lie further apart than the output's."""
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(2, 2, 16, "head", seed=19)
    ctx = cache.context(4)
    try:
        sfi.sfi_set_rope(ctx.handle, 128)
        p = cache.K.data_ptr()
        for new, qb, qt in ((1, 1024, 512), (3, 3 * 512, 1024), (3, 3 * 1024, 1024), (3, 512, 3 * 512)):
            a = dict(q=p, qb=qb, qt=qt, k=p, kb=256, kt=256, v=p, vb=256, vt=256, ctx_len=p, n_new=p, pos=p, max_new=new, q_out=p, K=p, V=p)
            assert sfi.load_library().sfi_rope_append(ctx.handle, *a.values(), None) == -1, (new, qb, qt)
    finally:
        ctx.close()
