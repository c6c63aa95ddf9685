"""sfi_rope_append against the formula in 64 bits: layouts, lengths, parts of a head, scalings, far positions, padding."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64

pytestmark = pytest.mark.gpu

TURNS = dict(kind="turns", factor=8.0, low=1.0, high=4.0, orig_ctx=8192)
DIMS = dict(kind="dims", factor=4.0, low=1.0, high=32.0, orig_ctx=4096)


def _step(msg):
    print(f"[gpu-rope] {msg}", flush=True)


def _check(got_bits, want, size):
    """One rounding to bf16 (half a step: 2^-8 of the value), fp32 products and sine / cosine before it (a few 2^-24 of the terms' sizes)."""
    slack = size * 2.0 ** -21
    bound = (np.abs(want) + slack) * 2.0 ** -8 + slack
    assert (np.abs(to64(got_bits) - want) <= bound).all()


def _run(B, T, Hq, Hkv, rot, interleaved, layout, rows, lens, n_new, pos, scaling=None, base=10000.0, magnitude=1.0, fused=True, with_q=True,
         in_place=False, page=16, seed=0):
    import torch
    import paper_2603_12038_amd as sfi

    g = torch.Generator().manual_seed(seed + 1)
    cache = ref.Cache(B, Hkv, rows, layout, page=page, seed=seed)
    before = [cache.numpy(0), cache.numpy(1)]
    ctx = cache.context(Hq)
    try:
        sfi.sfi_set_rope(ctx.handle, rot, base, interleaved=interleaved, scaling=scaling, magnitude=magnitude)
        if fused:
            qkv = torch.randn((B, T, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).cuda()
            q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
        else:
            q, k, v = (torch.randn((B, T, h, 128), generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
        q64, k64, v_bits = to64(bits(q)), to64(bits(k)), bits(v)
        q_out = q if in_place else torch.full((B, T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        _step(f"B={B} T={T} heads {Hq}/{Hkv} rot {rot} {layout} lens {lens} new {n_new} pos {pos}")
        sfi.sfi_rope_append(ctx.handle, q if with_q else None, k, v, i32(lens), None if n_new is None else i32(n_new),
                            None if pos is None else i32(pos), q_out if with_q else None, cache.K, cache.V)
        torch.cuda.synchronize()
        f = ref.freqs(rot, base, scaling)
        after = [cache.numpy(0), cache.numpy(1)]
        got_q = bits(q_out)
        for b in range(B):
            n = T if n_new is None else n_new[b]
            r0 = lens[b] - n
            at = np.arange(n) + (r0 if pos is None else pos[b])
            qr, qs = ref.rotate(q64[b, :n], at, f, interleaved, magnitude)
            kr, ks = ref.rotate(k64[b, :n], at, f, interleaved, magnitude)
            if with_q:
                _check(got_q[b, :n], qr, qs)
                if not in_place:
                    assert (got_q[b, n:] == bits(torch.tensor([7.0], dtype=torch.bfloat16))[0]).all(), "padding was written"
            _check(after[0][b, :, r0:lens[b]].transpose(1, 0, 2), kr, ks)
            assert np.array_equal(after[0][b, :, r0:lens[b], rot:].transpose(1, 0, 2), bits(k)[b, :n, :, rot:]), "part that is not turned"
            assert np.array_equal(after[1][b, :, r0:lens[b]].transpose(1, 0, 2), v_bits[b, :n])
            for w in (0, 1):  # no other row has changed
                assert np.array_equal(after[w][b, :, :r0], before[w][b, :, :r0])
                assert np.array_equal(after[w][b, :, lens[b]:], before[w][b, :, lens[b]:])
        assert sfi.sfi_device_status(ctx.handle) == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("layout", ref.LAYOUTS)
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rot", [16, 96, 128])
def test_a_token_and_a_prompt(layout, interleaved, rot):
    _run(3, 1, 8, 2, rot, interleaved, layout, 77, [77, 1, 33], None, None)
    _run(2, 19, 5, 1, rot, interleaved, layout, 40, [19, 40], None, None, fused=False, seed=2)


@pytest.mark.parametrize("scaling, magnitude", [(None, 1.0), (dict(kind="linear", factor=3.0), 0.5), (TURNS, 1.0), (DIMS, 1.1386)])
def test_scalings_and_far_positions(scaling, magnitude):
    """Positions up to the end of the 32-bit range: the angle keeps its fraction of a turn."""
    _run(4, 3, 4, 2, 64, False, "head", 50, [50, 3, 20, 8], [3, 3, 2, 1], [0, 131071, 9999991, 2147483600], scaling, 500000.0, magnitude)


def test_ragged_new_rows_with_none_and_with_all():
    _run(5, 33, 7, 7, 128, False, "thd", 70, [40, 33, 70, 9, 5], [0, 33, 1, 9, 4], None, page=32)


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (16, 1), (64, 8), (6, 3)])
def test_head_counts(Hq, Hkv):
    _run(2, 5, Hq, Hkv, 128, False, "head", 9, [9, 5], None, [100, 7])


def test_one_long_prompt_on_large_strides():
    _run(1, 2053, 4, 2, 128, True, "token", 2100, [2060], None, None)


def test_queries_in_place_and_without_queries():
    _run(3, 4, 8, 2, 128, False, "head", 30, [30, 4, 9], None, None, fused=False, in_place=True)
    _run(3, 4, 8, 2, 32, True, "head", 30, [30, 4, 9], None, None, with_q=False)


def test_freqs_given():
    import torch
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(1, 1, 8, "head")
    ctx = cache.context(1)
    try:
        f = [0.25, -1.5, 7.0, 0.0, 1e-7, 3.0, 100.0, 0.5]
        sfi.sfi_set_rope(ctx.handle, 16, freqs=f)
        x = torch.randn((1, 8, 1, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
        sfi.sfi_rope_append(ctx.handle, None, x, x, i32([8]), None, i32([5]), None, cache.K, cache.V)
        torch.cuda.synchronize()
        want, size = ref.rotate(to64(bits(x))[0], np.arange(8) + 5, f, False, 1.0)
        _check(cache.numpy(0)[0].transpose(1, 0, 2), want, size)
    finally:
        ctx.close()


def test_values_that_are_no_numbers_stay_in_their_pair():
    import torch
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(1, 1, 4, "head", seed=9)
    ctx = cache.context(1)
    try:
        sfi.sfi_set_rope(ctx.handle, 128)
        k = torch.randn((1, 1, 1, 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
        k[0, 0, 0, 3], k[0, 0, 0, 70] = float("nan"), float("inf")
        k = k.cuda()
        sfi.sfi_rope_append(ctx.handle, None, k, k, i32([3]), None, None, None, cache.K, cache.V)
        torch.cuda.synchronize()
        got = to64(cache.numpy(0)[0, 0, 2])
        bad = set(np.nonzero(~np.isfinite(got))[0].tolist())
        assert {3, 67} <= bad <= {3, 67, 6, 70}
        assert np.array_equal(cache.numpy(1)[0, 0, 2], bits(k)[0, 0, 0])
    finally:
        ctx.close()


def test_inputs_out_of_range_are_clamped_and_reported():
    """A count above the context or the batch of new rows, a negative one, a length above max_ctx; a block that is not in the pool takes no row."""
    import torch
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(4, 2, 32, "htd", seed=5)
    ctx = cache.context(4)
    try:
        sfi.sfi_set_rope(ctx.handle, 128)
        x = torch.randn((4, 4, 2, 128), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
        before = cache.numpy(1)
        _step("counts and lengths out of range")
        sfi.sfi_rope_append(ctx.handle, None, x, x, i32([2, 10, 99, -3]), i32([4, -1, 9, 1]), None, None, cache.K, cache.V)
        torch.cuda.synchronize()
        assert sfi.sfi_device_status(ctx.handle) == sfi.binding.GUARD_CTX_LEN | sfi.binding.GUARD_N_NEW
        after = cache.numpy(1)
        assert np.array_equal(after[0, :, :2].transpose(1, 0, 2), bits(x)[0, :2]) and np.array_equal(after[0, :, 2:], before[0, :, 2:])
        assert np.array_equal(after[1], before[1]) and np.array_equal(after[3], before[3])
        assert np.array_equal(after[2, :, 28:].transpose(1, 0, 2), bits(x)[2]) and np.array_equal(after[2, :, :28], before[2, :, :28])
        _step("a block id out of range")
        before, store = cache.numpy(1), [t.clone() for t in cache.store]
        wrong = cache.table.clone()
        wrong[1, 0] = cache.n_blocks + 5
        sfi.sfi_set_block_table(ctx.handle, wrong, cache.n_blocks)
        sfi.sfi_rope_append(ctx.handle, None, x, x, i32([0, 18, 0, 0]), i32([0, 4, 0, 0]), None, None, cache.K, cache.V)
        torch.cuda.synchronize()
        assert sfi.sfi_device_status(ctx.handle) == sfi.binding.GUARD_BLOCK
        after = cache.numpy(1)
        assert np.array_equal(after[1, :, 16:18].transpose(1, 0, 2), bits(x)[1, 2:]) and np.array_equal(after[1, :, :16], before[1, :, :16])
        changed = sum(int((a.view(torch.int16) != b.view(torch.int16)).flatten(1).any(1).sum()) for a, b in zip(cache.store, store))
        assert changed == 2, "rows went into a block that is not theirs"
    finally:
        ctx.close()


def test_another_stream():
    import torch
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(2, 2, 16, "head", seed=7)
    ctx = cache.context(4)
    try:
        s = torch.cuda.Stream()
        x = torch.randn((2, 3, 2, 128), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
        lens = i32([16, 3])
        torch.cuda.synchronize()
        sfi.sfi_set_rope(ctx.handle, 128, stream=s)
        sfi.sfi_rope_append(ctx.handle, None, x, x, lens, None, None, None, cache.K, cache.V, stream=s)
        s.synchronize()
        want, size = ref.rotate(to64(bits(x))[0], np.arange(3) + 13, ref.freqs(128, 10000.0), False, 1.0)
        _check(cache.numpy(0)[0, :, 13:].transpose(1, 0, 2), want, size)
    finally:
        ctx.close()


def test_refusals_with_a_rule():
    """Host-side checks of a context that has a rule: nothing is launched."""
    import paper_2603_12038_amd as sfi

    cache = ref.Cache(2, 2, 16, "head")
    ctx = cache.context(4)
    try:
        sfi.sfi_set_rope(ctx.handle, 128)
        p = cache.K.data_ptr()
        good = dict(q=p, qb=1024, qt=1024, k=p, kb=256, kt=256, v=p, vb=256, vt=256, ctx_len=p, n_new=p, pos=p, max_new=1, q_out=p, K=p, V=p)
        for over, code in ((dict(q=None), -1), (dict(q_out=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(ctx_len=None), -1), (dict(K=None), -1),
                           (dict(max_new=0), -1), (dict(max_new=17), -1), (dict(qb=-8), -1), (dict(kt=4), -4), (dict(vb=12), -4), (dict(q=p + 8), -4),
                           (dict(v=p + 2), -4), (dict(q_out=p + 4), -4), (dict(ctx_len=p + 2), -4), (dict(n_new=p + 1), -4), (dict(pos=p + 3), -4)):
            assert sfi.load_library().sfi_rope_append(ctx.handle, *{**good, **over}.values(), None) == code, over
    finally:
        ctx.close()
