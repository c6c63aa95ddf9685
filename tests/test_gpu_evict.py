"""sfi_evict: which rows stay (exactly), and where they and what belongs to them go, into another cache and in place."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import i32

pytestmark = pytest.mark.gpu


def _step(msg):
    print(f"[gpu-evict] {msg}", flush=True)


def _weights(rng, shape, kind):
    if kind == "plain":
        return np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":  # few values, zeros, negatives, infinities, NaN, denormals
        return rng.choice(np.array([0.0, -0.0, 1.0, 1.0, 2.5, -3.0, np.inf, -np.inf, np.nan, 1e-42, 1e-38, 3e38], np.float32), shape)
    if kind == "equal":
        return np.full(shape, 0.125, np.float32)
    return np.zeros(shape, np.float32)


def _run(B, Hkv, lens, budget, n_sink=4, recent=16, src="head", dst="head", in_place=False, rows_out=None, kind="plain", max_len=0, page=16,
         page_out=16, same_len=False, selector=None, seed=0, with_pos=True, with_weights_out=True):
    import torch
    import paper_2603_12038_amd as sfi

    rng = np.random.default_rng(seed)
    rows = max(max(lens), 1) + 7
    most = min(max_len or rows, n_sink + recent + budget)
    a = ref.Cache(B, Hkv, rows, src, page=page, seed=seed)
    ctx_a = a.context(Hkv, n_sink=n_sink, recent=recent, budget=budget, selector=selector)
    b = a if in_place else ref.Cache(B, Hkv, (rows_out or most + 5), dst, page=page_out, seed=seed + 1)
    ctx_b = ctx_a if in_place else b.context(Hkv, n_sink=0, recent=0, budget=0)
    try:
        w = _weights(rng, (B, Hkv, rows), kind)
        pos = rng.integers(0, 1 << 30, (B, Hkv, rows)).astype(np.int32)
        w_d, pos_d, len_d = torch.from_numpy(w).cuda(), torch.from_numpy(pos).cuda(), i32(lens)
        if in_place:
            w_out, pos_out, len_out = w_d, pos_d, len_d
        else:
            w_out = torch.full((B, Hkv, b.rows), 9.0, device="cuda")
            pos_out = torch.full((B, Hkv, b.rows), -9, dtype=torch.int32, device="cuda")
            len_out = len_d if same_len else i32([-9] * B)
        rs = i32([-9] * B)
        kept = torch.full((B, Hkv, max(budget, 1)), -9, dtype=torch.int32, device="cuda")
        n_kept = torch.full((B, Hkv), -9, dtype=torch.int32, device="cuda")
        old = [a.numpy(0), a.numpy(1)]
        out_before = [b.numpy(0), b.numpy(1)]
        _step(f"B={B} Hkv={Hkv} lens={lens[:6]} budget={budget} sink={n_sink} recent={recent} {src}->{'same' if in_place else dst} {kind}")
        sfi.sfi_evict(ctx_a.handle, a.K, a.V, len_d, max_len, budget, w_d, pos_d if with_pos else None, ctx_b.handle, b.K, b.V, len_out, rs,
                      w_out if with_weights_out else None, pos_out if with_pos else None, kept if budget else None, n_kept)
        torch.cuda.synchronize()
        new = [b.numpy(0), b.numpy(1)]
        kept, n_kept, len_out, rs = kept.cpu().numpy(), n_kept.cpu().numpy(), len_out.cpu().numpy(), rs.cpu().numpy()
        w_got, pos_got = w_out.cpu().numpy(), pos_out.cpu().numpy()
        for s in range(B):
            for h in range(Hkv):
                stay, middle = ref.kept_rows(w[s, h], lens[s], n_sink, recent, budget)
                n = len(stay)
                assert n_kept[s, h] == len(middle) and len_out[s] == n
                if budget:
                    assert np.array_equal(kept[s, h, :len(middle)], middle) and (kept[s, h, len(middle):budget] == -1).all()
                for i in (0, 1):
                    assert np.array_equal(new[i][s, h, :n], old[i][s, h, stay]), (s, h, i)
                    if not in_place:
                        assert np.array_equal(new[i][s, h, n:], out_before[i][s, h, n:]), "a row behind the last one was written"
                if with_weights_out:
                    assert np.array_equal(w_got[s, h, :n].view(np.uint32), w[s, h, stay].view(np.uint32)) and not w_got[s, h, n:].any()
                if with_pos:
                    assert np.array_equal(pos_got[s, h, :n], pos[s, h, stay])
                    assert in_place or (pos_got[s, h, n:] == -9).all()
            assert rs[s] == max(n_sink, len_out[s] - recent)
        if in_place:  # rows that were not in use are not touched
            for s in range(B):
                for i in (0, 1):
                    assert np.array_equal(new[i][s, :, lens[s]:], old[i][s, :, lens[s]:])
        assert sfi.sfi_device_status(ctx_a.handle) == 0
    finally:
        ctx_a.close()
        if not in_place:
            ctx_b.close()


@pytest.mark.parametrize("src, dst", [("head", "head"), ("token", "wide"), ("htd", "head"), ("head", "thd"), ("thd", "htd")])
@pytest.mark.parametrize("kind", ["plain", "ties"])
def test_into_another_cache(src, dst, kind):
    _run(3, 2, [700, 333, 81], 60, src=src, dst=dst, kind=kind, page_out=64)


@pytest.mark.parametrize("layout", ref.LAYOUTS)
@pytest.mark.parametrize("budget", [1, 130, 500])
def test_in_place(layout, budget):
    _run(3, 3, [1000, 517, 90], budget, src=layout, in_place=True, page=32)


@pytest.mark.parametrize("lens", [[0, 1, 3, 4], [5, 19, 20, 21], [22, 200, 0, 85]])
@pytest.mark.parametrize("in_place", [False, True])
def test_short_contexts_and_empty_slots(lens, in_place):
    """Nothing in the cache, less than the sink rows, nothing to rank, one row to rank, one more than the budget."""
    _run(4, 2, lens, 64, in_place=in_place, kind="ties")


@pytest.mark.parametrize("n_sink, recent, budget", [(0, 0, 7), (0, 5, 0), (9, 0, 1), (300, 4, 10), (4, 300, 10), (0, 0, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_odd_splits_of_the_context(n_sink, recent, budget, in_place):
    _run(2, 1, [260, 301], budget, n_sink=n_sink, recent=recent, in_place=in_place)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "none"])
@pytest.mark.parametrize("in_place", [False, True])
def test_long_contexts(kind, in_place):
    """More than 16384 rows to rank (three launches select), lengths on both sides of that within one call."""
    _run(2, 2, [20021, 900], 3001, recent=130, kind=kind, in_place=in_place, src="htd")


@pytest.mark.parametrize("n", [4096, 8192, 16384, 16385])
def test_lengths_where_the_selecting_launch_changes(n):
    _run(1, 2, [n + 20], 777, kind="ties")


@pytest.mark.parametrize("n, kind", [(16385, "ties"), (20011, "plain"), (32768, "equal"), (32769, "plain")])
def test_long_contexts_of_many_heads(n, kind):
    """64 pairs: one selecting launch up to 32768 rows between sink and recent rows, several behind them."""
    _run(1, 64, [n + 20], 301, kind=kind)


@pytest.mark.parametrize("n_sink", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_that_begin_anywhere_in_memory(n_sink, in_place):
    """Weights of J at every offset from 16 bytes, with one to nine positions of them."""
    _run(9, 3, [n_sink + 6 + i for i in range(1, 10)], 3, n_sink=n_sink, recent=6, in_place=in_place)
    _run(3, 3, [n_sink + 6 + 1021, n_sink + 6 + 258, n_sink + 6 + 4], 100, n_sink=n_sink, recent=6, in_place=in_place, kind="ties")


def test_many_rows_move_in_place():
    """Thousands of chunks over the rows of others: what is overwritten has been read."""
    _run(8, 8, [6000 - 17 * i for i in range(8)], 3500, recent=64, in_place=True, src="head")
    _run(2, 8, [12000, 11999], 5900, recent=0, n_sink=0, in_place=True, src="thd", page=64)


def test_a_bound_on_the_lengths_and_lengths_overwritten():
    _run(2, 2, [400, 350], 50, max_len=400, same_len=True)
    _run(2, 2, [40, 35], 300, max_len=40, rows_out=40)  # min(max_len, ...) rows have to fit


def test_without_positions_or_weights_out():
    _run(2, 2, [400, 350], 50, with_pos=False, with_weights_out=False)


def test_a_context_of_the_full_selector():
    sel = dict(gamma=0.5, beta=1.0, p=2.0, eta=0.5, lambda_clip=0.02, alpha_soft=0.5, alpha_cross=0.35, temp=1.0, eps=1e-8, nms_radius=2)
    _run(2, 2, [500, 350], 50, selector=sel)
    _run(1, 2, [17000], 500, selector=sel, in_place=True)


def test_twice_in_a_row_in_place_and_replayed():
    """A cache that has been cut is cut again; then both cuts as a captured graph, replayed on fresh copies."""
    import torch
    import paper_2603_12038_amd as sfi

    a = ref.Cache(2, 4, 900, "head", seed=11)
    ctx = a.context(4, n_sink=4, recent=16, budget=600)
    try:
        rng = np.random.default_rng(12)
        w0 = torch.from_numpy(_weights(rng, (2, 4, 900), "plain")).cuda()
        first = [t.clone() for t in a.store]
        w, lens = w0.clone(), i32([900, 611])
        kept, n_kept = torch.zeros((2, 4, 600), dtype=torch.int32, device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda")

        def reset():
            for t, f in zip(a.store, first):
                t.copy_(f)
            w.copy_(w0)
            lens.copy_(i32([900, 611]))

        def cuts():
            for budget in (500, 123):
                sfi.sfi_evict(ctx.handle, a.K, a.V, lens, 0, budget, w, None, ctx.handle, a.K, a.V, lens, None, w, None, kept, n_kept)

        reset()
        cuts()
        torch.cuda.synchronize()
        want = [t.clone() for t in a.store] + [w.clone(), lens.clone(), n_kept.clone(), kept.clone()]
        assert lens.tolist() == [143, 143]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            g.capture_begin()
            cuts()
            g.capture_end()
        torch.cuda.current_stream().wait_stream(s)
        for i in range(4):
            _step(f"replay {i}")
            reset()
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip([*a.store, w, lens, n_kept, kept], want):
                assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y)
    finally:
        ctx.close()


def test_lengths_out_of_range_are_clamped_and_reported():
    import torch
    import paper_2603_12038_amd as sfi

    a, b = ref.Cache(3, 1, 200, "head", seed=13), ref.Cache(3, 1, 100, "head", seed=14)
    ctx_a, ctx_b = a.context(1, n_sink=2, recent=8, budget=40), b.context(1, n_sink=2, recent=8, budget=40)
    try:
        w = torch.rand((3, 1, 200), generator=torch.Generator().manual_seed(1)).cuda()
        n_kept, kept = torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.zeros((3, 1, 40), dtype=torch.int32, device="cuda")
        out = i32([0, 0, 0])
        sfi.sfi_evict(ctx_a.handle, a.K, a.V, i32([999, -4, 30]), 150, 40, w, None, ctx_b.handle, b.K, b.V, out, None, None, None, kept, n_kept)
        torch.cuda.synchronize()
        assert sfi.sfi_device_status(ctx_a.handle) == sfi.binding.GUARD_CTX_LEN
        assert out.tolist() == [50, 0, 30]
        stay, _ = ref.kept_rows(w[0, 0].cpu().numpy(), 150, 2, 8, 40)
        assert np.array_equal(b.numpy(0)[0, 0, :50], a.numpy(0)[0, 0, stay])
    finally:
        ctx_a.close()
        ctx_b.close()
