"""sfi_weight_attn against attention in 64 bits: outputs, and every row's running weight."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64

pytestmark = pytest.mark.gpu
FULL = dict(gamma=0.5, beta=1.0, p=2.0, eta=0.5, lambda_clip=0.02, alpha_soft=0.5, alpha_cross=0.35, temp=1.0, eps=1e-8, nms_radius=2)


def _step(msg):
    print(f"[gpu-weigh] {msg}", flush=True)


def _run(B, Hq, Hkv, lens, layout="head", decay=1.0, given=True, same=False, bf16=False, max_len=0, support=True, seed=0, page=16, **ctx_more):
    import torch
    import paper_2603_12038_amd as sfi

    rows = max(lens) + 9
    g = torch.Generator().manual_seed(seed + 100)
    c = ref.Cache(B, Hkv, rows, layout, page=page, seed=seed)
    if support:
        heavy = (torch.rand(c.store[0].shape[:-1], generator=g) < 0.02).cuda()
        c.store[0].mul_((1 + 3 * heavy).to(torch.bfloat16).unsqueeze(-1))
    ctx = c.context(Hq, out_bf16=bf16, **ctx_more)
    try:
        q = torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).cuda()
        w = (torch.rand((B, Hkv, rows), generator=g) * 0.1).cuda()
        w[:, :, max(lens):] = float("nan")  # nothing to do with rows that are not there
        w_out = w if same else torch.full_like(w, 5.0)
        w0 = w.cpu().numpy().copy()
        out = torch.full((B, Hq, 128), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} lens={lens[:6]} {layout} decay={decay}")
        sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, i32(lens), max_len, decay, w if given else None, w_out, out)
        torch.cuda.synchronize()
        K, V, qn = to64(c.numpy(0)), to64(c.numpy(1)), to64(bits(q))
        got, w_got = out.float().cpu().numpy().astype(np.float64), w_out.cpu().numpy()
        for b, n in enumerate(lens):
            want, p, size = ref.attend(qn[b], K[b, :, :n], V[b, :, :n])
            assert (np.abs(got[b] - want) <= ref.out_bound(p, V[b, :, :n], Hq, size, want, bf16)).all(), b
            share = p.reshape(Hkv, Hq // Hkv, n).mean(1)
            total = share + (decay * w0[b, :, :n].astype(np.float64) if given else 0.0)
            bound = 2 * ref.weight_slack(size) * share + 2.0 ** -22 * total + 1e-37
            assert (np.abs(w_got[b, :, :n] - total) <= bound).all(), b
            rest = w0[b, :, n:] if same else np.full_like(w0[b, :, n:], 5.0)
            assert np.array_equal(w_got[b, :, n:], rest, equal_nan=True), "a row behind the context was touched"
        assert sfi.sfi_device_status(ctx.handle) == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("layout", ref.LAYOUTS)
@pytest.mark.parametrize("Hq, Hkv", [(2, 2), (10, 2), (16, 1), (7, 1)])
def test_layouts_and_groups(layout, Hq, Hkv):
    _run(3, Hq, Hkv, [130, 1, 517], layout=layout, decay=0.9)


@pytest.mark.parametrize("lens", [[0, 1, 0, 2], [31, 32, 33, 0], [1023, 1024, 1025, 2049]])
@pytest.mark.parametrize("same", [False, True])
def test_short_lengths_and_empty_slots(lens, same):
    _run(4, 8, 2, lens, same=same, decay=0.5)


@pytest.mark.parametrize("B, n", [(1, 9000), (2, 5003), (6, 3001)])
@pytest.mark.parametrize("bf16", [False, True])
def test_longer_contexts(B, n, bf16):
    _run(B, 8, 2, [n - 401 * i for i in range(B)], bf16=bf16, layout="thd", page=64, support=False)


def test_without_weights_before_and_with_a_bound():
    _run(2, 4, 2, [300, 50], given=False)
    _run(2, 4, 2, [300, 50], max_len=301)
    _run(2, 4, 2, [300, 50], decay=0.0)


def test_whatever_the_context_selects_with():
    """Sink, recent window, selector and power mean of the context have no part in the weights."""
    _run(2, 8, 2, [700, 40], n_sink=100, recent=500, selector=FULL, alpha=0.5)
    _run(2, 8, 2, [700, 40], n_sink=0, recent=0)


def test_few_rows_of_like_weight_lose_nothing_to_one_side():
    """27 rows: the output's error has no common direction (weights cut off at 16 bits would all be 6e-6 too small)."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, n = 4, 16, 4, 27
    c = ref.Cache(B, Hkv, n, "head", seed=3)
    c.store[1].abs_()
    ctx = c.context(Hq)
    try:
        q = (0.3 * torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(4))).to(torch.bfloat16).cuda()
        w, out = torch.zeros((B, Hkv, n), device="cuda"), torch.zeros((B, Hq, 128), device="cuda")
        sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, i32([n] * B), 0, 1.0, None, w, out)
        torch.cuda.synchronize()
        K, V, qn = to64(c.numpy(0)), to64(c.numpy(1)), to64(bits(q))
        off = [(out[b].cpu().numpy() - r) / r for b in range(B) for r in [ref.attend(qn[b], K[b], V[b])[0]]]
        # each weight is off by at most 2^-17, either way, of 27 in each of 8192 outputs: their mean is far below that
        assert abs(float(np.mean(off))) < 2.0 ** -20
    finally:
        ctx.close()


def test_weights_add_up_over_steps_in_place():
    import torch
    import paper_2603_12038_amd as sfi

    c = ref.Cache(2, 2, 90, "head", seed=21)
    ctx = c.context(8)
    try:
        g = torch.Generator().manual_seed(22)
        w, out, lens = torch.zeros((2, 2, 90), device="cuda"), torch.zeros((2, 8, 128), device="cuda"), i32([60, 7])
        K = to64(c.numpy(0))
        want = np.zeros((2, 2, 90))
        V = to64(c.numpy(1))
        size = 0.0
        for t in range(6):
            q = torch.randn((2, 8, 128), generator=g).to(torch.bfloat16).cuda()
            sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, lens, 0, 0.75, w, w, out)
            for b, n in enumerate((60 + t, 7 + t)):
                p, s = ref.attend(to64(bits(q))[b], K[b, :, :n], V[b, :, :n])[1:]
                want[b, :, :n] = 0.75 * want[b, :, :n] + p.reshape(2, 4, n).mean(1)
                size = max(size, s)
            lens += 1
        torch.cuda.synchronize()
        assert (np.abs(w.cpu().numpy() - want) <= (2 * ref.weight_slack(size) + 2.0 ** -21) * want + 1e-37).all()
    finally:
        ctx.close()


def test_a_slow_step_on_the_same_context_is_what_it_was():
    import torch
    import paper_2603_12038_amd as sfi

    c = ref.Cache(2, 2, 800, "head", seed=31)
    ctx = c.context(8, budget=100)
    try:
        q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(32)).to(torch.bfloat16).cuda()
        w, out, lens = torch.zeros((2, 2, 800), device="cuda"), torch.zeros((2, 8, 128), device="cuda"), i32([800, 333])

        def slow():
            o, sel, n = torch.zeros_like(out), torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
            sfi.sfi_slow_step(ctx.handle, q, c.K, c.V, lens, 0, 100, o, sel, n)
            torch.cuda.synchronize()
            return o, sel, n

        a = slow()
        sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, lens, 0, 1.0, None, w, out)
        b = slow()
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    finally:
        ctx.close()
