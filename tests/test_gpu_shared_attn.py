"""sfi_shared_attn against attention in 64 bits: rows of the lead, then the sequence's own; what is not used may hold anything."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64

pytestmark = pytest.mark.gpu


def _step(msg):
    print(f"[gpu-shared] {msg}", flush=True)


def _run(B, Hq, Hkv, lens, shared, lead=0, layout="head", max_shared=None, max_len=0, bf16=False, seed=0, page=16, poison=True, scale=0.0,
         status=0, alias=False):
    """poison: NaN in every row that is not to be used.  alias: the table entries of wholly shared blocks name the lead's blocks."""
    import torch
    import paper_2603_12038_amd as sfi

    rows = max(max(lens), 1) + 40
    g = torch.Generator().manual_seed(seed + 200)
    c = ref.Cache(B, Hkv, rows, layout, page=page, seed=seed)
    cap = max_len or rows
    L = [min(max(n, 0), cap) for n in lens]
    top = max(s for s in shared) if max_shared is None else max_shared
    S = [min(max(s, 0), n, L[lead], top) for s, n in zip(shared, L)]
    heavy = (torch.rand(c.store[0].shape[:-1], generator=g) < 0.02).cuda()
    c.store[0].mul_((1 + 3 * heavy).to(torch.bfloat16).unsqueeze(-1))
    if alias:
        assert c.paged
        for b in range(B):
            c.table_np[b, :S[b] // page] = c.table_np[lead, :S[b] // page]
        c.table.copy_(torch.from_numpy(c.table_np))
    K, V = to64(c.numpy(0)), to64(c.numpy(1))
    if poison and not alias:
        nan = np.full((Hkv, 128), 0x7FC1, np.uint16)
        for b in range(B):
            used = np.zeros(rows, bool)
            used[S[b]:L[b]] = True
            if b == lead:
                used[:max(S)] = True
            for t in (0, 1):
                view = (c.K, c.V)[t]
                for r in np.nonzero(~used)[0] if rows <= 400 else [r for r in (0, 1, S[b] - 1, L[b], L[b] + 1, rows - 1) if 0 <= r < rows and not used[r]]:
                    c.put(t, b, int(r), nan)
    ctx = c.context(Hq, out_bf16=bf16, scale=scale)
    try:
        q = torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).cuda()
        out = torch.full((B, Hq, 128), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} lens={lens[:6]} shared={shared[:6]} lead={lead} {layout} max_shared={top}")
        sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, i32(lens), i32(shared), lead, top, max_len, out)
        torch.cuda.synchronize()
        qn, got = to64(bits(q)), out.float().cpu().numpy().astype(np.float64)
        for b in range(B):
            k, v = (np.concatenate((x[lead, :, :S[b]], x[b, :, S[b]:L[b]]), axis=1) for x in (K, V))
            want, p, size = ref.attend(qn[b], k, v, scale or None)
            assert (np.abs(got[b] - want) <= ref.out_bound(p, v, Hq, size, want, bf16)).all(), b
        assert sfi.sfi_device_status(ctx.handle) == status
        return out
    finally:
        ctx.close()


@pytest.mark.parametrize("layout", ref.LAYOUTS)
@pytest.mark.parametrize("Hq, Hkv", [(2, 2), (10, 2), (16, 1)])
def test_layouts_and_groups(layout, Hq, Hkv):
    _run(5, Hq, Hkv, [200, 131, 96, 160, 97], [96, 96, 96, 96, 96], layout=layout)


@pytest.mark.parametrize("B, Hq, Hkv", [(1, 8, 2), (2, 8, 1), (4, 16, 2), (3, 33, 3), (9, 8, 1), (13, 13, 1), (33, 8, 1), (70, 16, 1)])
def test_numbers_of_query_columns(B, Hq, Hkv):
    """8 to 1120 columns a head: every width of the product and what is left over in the last block of columns."""
    _run(B, Hq, Hkv, [300 + i % 7 for i in range(B)], [293] * B)


@pytest.mark.parametrize("lead", [0, 3, 6])
@pytest.mark.parametrize("layout", ["head", "thd"])
def test_sequences_share_different_lengths(lead, layout):
    """None, one row, all of their rows, more than the lead's row would allow is asked elsewhere; own rows that begin inside a tile and a page."""
    lens = [300, 1, 64, 250, 199, 5, 231]
    shared = [0, 1, 64, 33, 198, 0, 100]
    n = lens[lead]
    _run(7, 4, 2, lens, [min(s, n) for s in shared], lead=lead, layout=layout)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 127, 128, 129, 255, 257])
def test_lengths_around_tiles(n):
    _run(4, 8, 2, [n, n + 1, n + 40, n], [n, n, n, n - 1])


def test_empty_slots_and_an_empty_lead():
    _run(4, 8, 2, [0, 50, 0, 3], [0, 0, 0, 0])
    _run(4, 8, 2, [40, 0, 50, 40], [40, 0, 40, 40])
    _run(3, 8, 2, [0, 0, 0], [0, 0, 0])


def test_nothing_shared_at_all():
    _run(3, 8, 2, [100, 333, 7], [0, 0, 0], max_shared=0)
    _run(3, 8, 2, [100, 333, 7], [0, 0, 0], max_shared=100)


@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("bf16", [False, True])
def test_longer_prefixes(layout, bf16):
    _run(6, 12, 3, [5003, 4100 + 11, 4100, 4500, 4101, 4200], [4100, 4100, 4100, 4099, 4100, 17], layout=layout, bf16=bf16, page=64, lead=0)


@pytest.mark.parametrize("B, Hq, Hkv, n", [(24, 32, 2, 2500), (40, 16, 2, 1500)])
def test_many_columns_over_longer_prefixes(B, Hq, Hkv, n):
    _run(B, Hq, Hkv, [n + 3 * i for i in range(B)], [n - (i % 3) * (n // 4) for i in range(B)])


def test_tables_that_name_the_same_blocks():
    for page in (16, 64):
        out = _run(5, 8, 2, [400, 321, 330, 390, 320], [320] * 5, layout="htd", page=page, alias=True)
        assert out.isfinite().all()


@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("B, Hq, Hkv, most", [(1, 8, 1, 6000), (3, 4, 2, 3000), (13, 8, 4, 1500), (40, 8, 4, 900), (100, 2, 1, 700), (130, 2, 1, 500)])
def test_own_rows_of_very_different_lengths(B, Hq, Hkv, most, layout):
    """None, a few, and many rows of their own, shared out to workgroups together; one sequence shares nothing."""
    own = [(i * 7919) % most if i % 3 else i % 5 for i in range(B)]
    own[B // 2] = most
    shared = [100 - (i % 4) * 3 for i in range(B)]
    shared[0] = 100
    if B > 2:
        shared[1] = 0
    _run(B, Hq, Hkv, [s + o for s, o in zip(shared, own)], shared, layout=layout, poison=B < 40)


def test_same_as_dense_attention_where_the_rows_are_the_same():
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, n, m = 6, 16, 4, 700, 90
    c = ref.Cache(B, Hkv, n + m, "head", seed=41)
    for t in c.store:
        t[1:, :, :n] = t[:1, :, :n]
    ctx = c.context(Hq)
    try:
        q = torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(42)).to(torch.bfloat16).cuda()
        lens = i32([n + 15 * i for i in range(B)])
        a, b = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hq, 128), device="cuda")
        sfi.sfi_dense_attn(ctx.handle, q, c.K, c.V, lens, 0, a)
        sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, lens, i32([n] * B), 2, n, 0, b)
        torch.cuda.synchronize()
        # both within the bound of the 64-bit result: 2 * slack of sum p |v| <= max |v|
        assert (a - b).abs().max().item() <= 4 * ref.weight_slack(40.0) * float(c.V.float().abs().max())
    finally:
        ctx.close()


def test_a_scale_and_peaked_softmax():
    _run(4, 8, 2, [150, 160, 170, 128], [128] * 4, scale=1.5)


@pytest.mark.parametrize("B, Hq, Hkv", [(3, 4, 2), (5, 5, 1), (6, 16, 1), (8, 32, 2), (20, 32, 2)])
@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("bad, own", [("nan", 1), ("inf", 1), ("nan", 500)])
def test_rows_that_only_others_share_may_hold_anything(B, Hq, Hkv, layout, bad, own):
    """Sequences that share less of the lead are not touched by what the rows behind their share hold, in K or in V."""
    import torch
    import paper_2603_12038_amd as sfi

    n, few = 700, [0, 1, 33, 416]
    c = ref.Cache(B, Hkv, n + own + 20, layout, seed=61)
    lens = [n + own + i % 9 for i in range(B)]
    shared = [n if b in (0, 1) else few[b % 4] for b in range(B)]
    K, V = to64(c.numpy(0)), to64(c.numpy(1))
    row = np.full((Hkv, 128), 0x7FC1 if bad == "nan" else 0x7F80, np.uint16)
    c.put(0, 0, 500, row), c.put(1, 0, 450, row), c.put(1, 0, 600, row)
    ctx = c.context(Hq)
    try:
        q = torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(62)).to(torch.bfloat16).cuda()
        out = torch.zeros((B, Hq, 128), device="cuda")
        _step(f"B={B} heads {Hq}/{Hkv} {layout} {bad}")
        sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, i32(lens), i32(shared), 0, n, 0, out)
        torch.cuda.synchronize()
        qn, got = to64(bits(q)), out.cpu().numpy().astype(np.float64)
        assert not np.isfinite(got[:2]).any()
        for b in range(2, B):
            k, v = (np.concatenate((x[0, :, :shared[b]], x[b, :, shared[b]:lens[b]]), axis=1) for x in (K, V))
            want, p, size = ref.attend(qn[b], k, v)
            assert (np.abs(got[b] - want) <= ref.out_bound(p, v, Hq, size, want, False)).all(), b
    finally:
        ctx.close()


def test_inputs_out_of_range_are_clamped_and_reported():
    _run(4, 8, 2, [200, 150, 100, 60], [200, 190, -5, 60], lead=1, max_shared=150, poison=False, status=32)
    _run(3, 8, 2, [200, 100, 90], [80, 80, 80], max_len=150, poison=False, status=1)


def test_outputs_repeat_and_replay():
    """The same bits every time: alone, next to another context on another stream, and replayed from a graph that two calls share."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv = 8, 32, 4
    c = ref.Cache(B, Hkv, 1300, "head", seed=51)
    ctx, ctx2 = c.context(Hq), c.context(Hq)
    try:
        g = torch.Generator().manual_seed(52)
        qs = [torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
        lens, sh = i32([1200 + 9 * i for i in range(B)]), i32([1100] * B)
        outs = [torch.zeros((B, Hq, 128), device="cuda") for _ in range(2)]

        def call(h, i, o):
            sfi.sfi_shared_attn(h, qs[i], c.K, c.V, lens, sh, 0, 1100, 0, o)

        for i in (0, 1):
            call(ctx.handle, i, outs[i])
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        s = torch.cuda.Stream()
        _step("two contexts, two streams")
        for _ in range(3):
            outs[0].zero_(), outs[1].zero_()
            s.wait_stream(torch.cuda.current_stream())
            call(ctx.handle, 0, outs[0])
            with torch.cuda.stream(s):
                call(ctx2.handle, 1, outs[1])
            torch.cuda.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
        graph = torch.cuda.CUDAGraph()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph.capture_begin()
            for i in (0, 1):
                call(ctx.handle, i, outs[i])
            graph.capture_end()
        torch.cuda.current_stream().wait_stream(s)
        for i in range(4):
            _step(f"replay {i}")
            outs[0].zero_(), outs[1].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    finally:
        ctx.close()
        ctx2.close()
