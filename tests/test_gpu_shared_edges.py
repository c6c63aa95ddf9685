"""sfi_shared_attn where it could answer wrongly without a word: what is no number stays none, weights keep their bits, bounds that are loose."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64
from test_gpu_shared_attn import _run

pytestmark = pytest.mark.gpu


def _step(msg):
    print(f"[gpu-shared-edges] {msg}", flush=True)


@pytest.mark.parametrize("B, Hq, Hkv", [(4, 4, 2), (8, 32, 2), (20, 32, 2), (66, 16, 2)])
@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("own", [3, 700])
@pytest.mark.parametrize("bf16", [False, True])
def test_what_is_no_number_stays_none(B, Hq, Hkv, layout, own, bf16):
    """A NaN that a sequence sees (a key of its own, one of the lead's, its query, one element of a value) comes out of it also where others
    share more of the lead, and the other sequences do not notice."""
    import torch
    import paper_2603_12038_amd as sfi

    n, nan = 300, np.full((Hkv, 128), 0x7FC1, np.uint16)
    c = ref.Cache(B, Hkv, n + own + 20, layout, seed=71)
    lens = [n + own + i % 9 for i in range(B)]
    shared = [n if b in (0, B - 1) else [40, 199, 200, 33][b % 4] for b in range(B)]
    shared[1] = 0
    c.put(0, 1, 20, nan)  # sequence 1 shares nothing: a key of its own
    value = np.zeros((Hkv, 128), np.uint16)
    value[:, 5] = 0x7FC1
    c.put(1, 2, lens[2] - 1, value)  # sequence 2: element 5 of its last value
    K, V = to64(c.numpy(0)), to64(c.numpy(1))
    ctx = c.context(Hq, out_bf16=bf16)
    try:
        q = torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(72)).to(torch.bfloat16)
        q[3, 1, 7] = float("nan") if B > 4 else q[3, 1, 7]  # sequence 3: one element of one head's query
        q = q.cuda()
        out = torch.zeros((B, Hq, 128), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} {layout} own {own} bf16 {bf16}")
        sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, i32(lens), i32(shared), 0, n, 0, out)
        torch.cuda.synchronize()
        qn, got = to64(bits(q)), out.float().cpu().numpy().astype(np.float64)
        for b in range(B):
            k, v = (np.concatenate((x[0, :, :shared[b]], x[b, :, shared[b]:lens[b]]), axis=1) for x in (K, V))
            bad = np.zeros((Hq, 128), bool)
            if b == 1:
                bad[:] = True
            elif b == 2:
                bad[:, 5] = True
            elif b == 3 and B > 4:
                bad[1] = True
            assert np.isnan(got[b][bad]).all(), f"sequence {b}: a number in place of NaN"
            want, p, size = ref.attend(np.nan_to_num(qn[b]), np.nan_to_num(k), np.nan_to_num(v))
            bound = ref.out_bound(p, np.nan_to_num(v), Hq, size, want, bf16)
            assert (np.abs(got[b] - want) <= bound)[~bad].all(), b
    finally:
        ctx.close()


def _two_terms_miss():
    """Query values x > 0 in bf16 whose weight 2^(-x log2(e) / sqrt(128)), beside one of 1, is off by at least 2^-18 of itself as the sum of two bf16 terms."""
    import torch

    x = torch.arange(1, 2048, dtype=torch.float32).mul_(2.0 ** -5).to(torch.bfloat16).unique().double()
    p = torch.exp(-x / 128.0 ** 0.5).float()
    hi = p.to(torch.bfloat16).float()
    lo = (p - hi).to(torch.bfloat16).float()
    return x[(((p - hi - lo).abs() / p) >= 2.0 ** -18) & (p > 0.02)]


def test_values_that_tell_two_terms_from_three():
    """(of the check below: it has values to work with)"""
    assert len(_two_terms_miss()) >= 16


# Half of the rows have a weight of 1 and values of 0, the others a weight p and values of 1: the output is p / (1 + p), and its error that of p
# in the products with V (the sums of the weights are in fp32).  In fp32 p is off by its exponent's two roundings (together below 7 2^-24: |exponent| < 6, times ln 2) and
# 2^-23 for the exponential; the sums of either side round a few times per tile, wave and record.  That is below 48 roundings of at most 2^-24, to either side:
# 2^-24 sqrt(48 / 3) = 2^-22 as a root of the mean square over columns of many p.  Two bf16 terms are off by 2^-18 or more in every column, and so is the
# output: 2^-20 lies between.
EXACT = 2.0 ** -20


@pytest.mark.parametrize("B, Hq, Hkv", [(2, 8, 1), (5, 16, 4), (6, 32, 2), (20, 16, 1), (17, 64, 4)])
@pytest.mark.parametrize("max_shared", [512, 24575, 24576, 30000])
@pytest.mark.parametrize("own", [0, 96])
def test_weights_keep_their_bits_behind_fp32_outputs(B, Hq, Hkv, max_shared, own):
    """8 to 320 columns a head, the bound of the shared rows exact and far too large: the same accuracy."""
    import torch
    import paper_2603_12038_amd as sfi

    n, rows = 512, max_shared + own + 8
    xs = _two_terms_miss()
    K = torch.zeros((1, 1, rows, 128), dtype=torch.bfloat16)
    V = torch.zeros((1, 1, rows, 128), dtype=torch.bfloat16)
    K[:, :, 1::2, 0], V[:, :, 1::2] = 1.0, 1.0
    K, V = (t.cuda().expand(B, Hkv, rows, 128) for t in (K, V))  # strides of zero: all sequences hold the same rows
    ctx = sfi.SfiContext(B, Hq, Hkv, rows, 64, 4, 64, K, V)
    try:
        x = xs[torch.arange(B * Hq) * 7919 % len(xs)].view(B, Hq)
        q = torch.zeros((B, Hq, 128), dtype=torch.bfloat16)
        q[:, :, 0] = -x.to(torch.bfloat16)
        q, out = q.cuda(), torch.zeros((B, Hq, 128), device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} bound {max_shared} own {own}")
        sfi.sfi_shared_attn(ctx.handle, q, K, V, i32([n + own] * B), i32([n] * B), 0, max_shared, 0, out)
        torch.cuda.synchronize()
        p = torch.exp(-x / 128.0 ** 0.5)
        want = (p / (1 + p))[:, :, None]
        off = out.cpu().double() / want - 1
        assert off.square().mean().sqrt().item() <= EXACT
    finally:
        ctx.close()


@pytest.mark.parametrize("layout", ["head", "token", "htd"])
@pytest.mark.parametrize("B, Hq, Hkv", [(17, 16, 1), (33, 32, 2), (41, 28, 4)])
@pytest.mark.parametrize("bf16", [True, False])
def test_more_than_256_columns(B, Hq, Hkv, layout, bf16):
    """272, 528 and 287 columns a head: the last group of 256 partly empty, shares of every length, tiles and stages cut anywhere."""
    n = 1100
    shared = [n - (i * 389) % (n + 1) for i in range(B)]
    shared[B // 2] = 0
    _run(B, Hq, Hkv, [max(s, 1) + (i * 53) % 70 for i, s in enumerate(shared)], shared, layout=layout, bf16=bf16, page=32)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B", [2, 17])
def test_bounds_far_above_the_lengths(B, bf16):
    """17 columns and more under a bound of max_ctx: the rows that are there decide, not the bound."""
    _run(B, 16, 1, [90 + i for i in range(B)], [90 - i for i in range(B)], max_shared=90 + B + 39 - 1, bf16=bf16)


@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("B", [4, 20])
def test_one_sequence_shares_nothing_under_a_tight_bound(B, layout):
    """max_shared close to max_len: rows of their own are read by one workgroup per pair, the whole of a sequence among them."""
    lens = [2000 + i % 7 for i in range(B)]
    shared = [1990] * B
    shared[1] = 0
    _run(B, 16, 8 if B == 4 else 2, lens, shared, layout=layout, max_shared=1990, max_len=2010)


@pytest.mark.parametrize("B, Hq, Hkv", [(3, 8, 2), (6, 16, 4), (20, 32, 2)])
def test_each_output_is_that_of_dense_attention(B, Hq, Hkv):
    """Element by element within what each of the two may be off by, where the first rows are the same.  Together they are closer: the dense
    launch cuts its weights off at two bf16 terms, 2^-17 too small in the mean, the rest is below that, so 2^-16 of the outputs as a root of the mean square;
    one row of 700 left out would be about 700^-1/2."""
    import torch
    import paper_2603_12038_amd as sfi

    n, m = 700, 90
    c = ref.Cache(B, Hkv, n + m, "head", seed=81)
    for t in c.store:
        t[1:, :, :n] = t[:1, :, :n]
    ctx = c.context(Hq)
    try:
        q = torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(82)).to(torch.bfloat16).cuda()
        L = [n + 4 * i for i in range(B)]
        a, b = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hq, 128), device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} dense and shared")
        sfi.sfi_dense_attn(ctx.handle, q, c.K, c.V, i32(L), 0, a)
        sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, i32(L), i32([n] * B), B - 1, n, 0, b)
        torch.cuda.synchronize()
        K, V, qn = to64(c.numpy(0)), to64(c.numpy(1)), to64(bits(q))
        a, b = (t.cpu().numpy().astype(np.float64) for t in (a, b))
        for i in range(B):
            want, p, size = ref.attend(qn[i], K[i, :, :L[i]], V[i, :, :L[i]])
            bound = ref.out_bound(p, V[i, :, :L[i]], Hq, size, want, False)
            assert (np.abs(a[i] - want) <= bound).all() and (np.abs(b[i] - want) <= bound).all() and (np.abs(a[i] - b[i]) <= 2 * bound).all(), i
        assert np.sqrt(((a - b) ** 2).mean() / (a ** 2).mean()) <= 2.0 ** -16
    finally:
        ctx.close()
