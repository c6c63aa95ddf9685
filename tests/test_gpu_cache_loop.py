"""The operators as a decode loop uses them: rows rotated and written, read and weighed, and dropped when the cache is full; a prompt that
a batch shares."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64

pytestmark = pytest.mark.gpu


def _step(msg):
    print(f"[gpu-loop] {msg}", flush=True)


@pytest.mark.parametrize("layout", ["head", "htd"])
def test_a_bounded_cache_over_many_steps(layout):
    """A prompt, then tokens one by one into a cache of 120 rows that is cut back to 4 + 40 + 16 whenever it is full.  A plain simulation in 64 bits
    keeps, per KV head, the list of positions that are left; which rows go follows the GPU's own weights, which are checked against it."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, cap, sink, recent, budget, prompt, steps = 2, 8, 2, 120, 4, 16, 40, 50, 200
    g = torch.Generator().manual_seed(61)
    c = ref.Cache(B, Hkv, cap, layout, seed=60, fill="nan")
    ctx = c.context(Hq, n_sink=sink, recent=recent, budget=budget)
    f = ref.freqs(64, 10000.0)
    try:
        sfi.sfi_set_rope(ctx.handle, 64)
        total = prompt + steps
        qkv = torch.randn((B, total, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).cuda()
        q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
        lens, pos = i32([prompt] * B), i32([0] * B)
        w = torch.zeros((B, Hkv, cap), device="cuda")
        row_pos = torch.full((B, Hkv, cap), -1, dtype=torch.int32, device="cuda")
        q_rot = torch.zeros((B, prompt, Hq, 128), dtype=torch.bfloat16, device="cuda")
        sfi.sfi_rope_append(ctx.handle, q[:, :prompt], k[:, :prompt], v[:, :prompt], lens, None, pos, q_rot, c.K, c.V)
        row_pos[:, :, :prompt] = torch.arange(prompt, device="cuda", dtype=torch.int32)
        rows = [[list(range(prompt)) for _ in range(Hkv)] for _ in range(B)]
        want_w = [[np.zeros(prompt) for _ in range(Hkv)] for _ in range(B)]
        q64 = to64(bits(q))
        k_bits = bits(k)
        k_rot = np.zeros((B, total, Hkv, 128))
        for b in range(B):
            k_rot[b] = ref.rotate(to64(k_bits[b]), np.arange(total), f, False, 1.0)[0]
        v64 = to64(bits(v))
        out, tok_q = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, 1, Hq, 128), dtype=torch.bfloat16, device="cuda")
        kept, n_kept = torch.zeros((B, Hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros((B, Hkv), dtype=torch.int32, device="cuda")
        n, cuts = prompt, 0
        for t in range(prompt, total):
            if n == cap:
                before = w.cpu().numpy()
                sfi.sfi_evict(ctx.handle, c.K, c.V, lens, 0, budget, w, row_pos, ctx.handle, c.K, c.V, lens, None, w, row_pos, kept, n_kept)
                for b in range(B):
                    for h in range(Hkv):
                        stay, _ = ref.kept_rows(before[b, h], n, sink, recent, budget)
                        rows[b][h] = [rows[b][h][r] for r in stay]
                        want_w[b][h] = want_w[b][h][stay]
                n = sink + budget + recent
                cuts += 1
                assert lens.tolist() == [n] * B
                for b in range(B):
                    for h in range(Hkv):
                        assert row_pos[b, h, :n].tolist() == rows[b][h]
            n += 1
            lens += 1
            pos.fill_(t)
            sfi.sfi_rope_append(ctx.handle, q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], lens, None, pos, tok_q, c.K, c.V)
            row_pos[:, :, n - 1] = t
            sfi.sfi_weight_attn(ctx.handle, tok_q.view(B, Hq, 128), c.K, c.V, lens, 0, 1.0, w, w, out)
            got_q = to64(bits(tok_q)).reshape(B, Hq, 128)
            got, w_now = out.cpu().numpy().astype(np.float64), w.cpu().numpy()
            for b in range(B):
                rq, size_q = ref.rotate(q64[b, t], np.full((), t), f, False, 1.0)
                assert (np.abs(got_q[b] - rq) <= (np.abs(rq) + size_q * 2.0 ** -21) * 2.0 ** -8 + size_q * 2.0 ** -21).all()
                for h in range(Hkv):
                    rows[b][h].append(t)
                    # keys as they were rounded into the cache: nearest bf16 of the rotated key
                    kk = torch.from_numpy(k_rot[b, rows[b][h], h]).to(torch.float32).to(torch.bfloat16)
                    kk = kk.to(torch.float64).numpy()[None]
                    vv = v64[b, rows[b][h], h][None]
                    G = Hq // Hkv
                    o, p, size = ref.attend(got_q[b, h * G:(h + 1) * G], kk, vv)
                    # a rotated key may have been rounded the other way where it lies on the border of two bf16 values: 2^-8 of one element of 128
                    # in a row, a logit of at most 2^-8 * |q| |k| * scale of that element
                    slack = 2 * ref.weight_slack(size) + 2 * 2.0 ** -8 * float(np.abs(got_q[b]).max() * np.abs(kk).max()) / 128 ** 0.5
                    assert (np.abs(got[b, h * G:(h + 1) * G] - o) <= slack * np.matmul(p, np.abs(vv[0])) + 1e-30).all(), (t, b, h)
                    want_w[b][h] = np.append(want_w[b][h], 0.0) + p.mean(0)
                    assert (np.abs(w_now[b, h, :n] - want_w[b][h]) <= (slack + 2.0 ** -20) * want_w[b][h] + 1e-37).all()
        assert cuts >= 3
        assert sfi.sfi_device_status(ctx.handle) == 0
    finally:
        ctx.close()


def test_a_prompt_that_a_batch_shares():
    """The lead writes a prompt; the others' tables name its blocks.  Everyone goes on by himself: appends, attention over shared and own rows, which is
    what dense attention gives over the same tables; then an eviction in place that leaves the shared rows (sink rows) where they are."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, page, prompt, own, recent, budget = 4, 8, 2, 16, 96, 40, 8, 12
    cap = prompt + own
    g = torch.Generator().manual_seed(71)
    c = ref.Cache(B, Hkv, cap, "htd", page=page, seed=70, fill="nan")
    for b in range(1, B):
        c.table_np[b, :prompt // page] = c.table_np[0, :prompt // page]
    c.table.copy_(torch.from_numpy(c.table_np))
    ctx = c.context(Hq, n_sink=prompt, recent=recent, budget=budget)
    try:
        sfi.sfi_set_rope(ctx.handle, 128, interleaved=True)
        qkv = torch.randn((B, prompt, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).cuda()
        _, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
        sfi.sfi_rope_append(ctx.handle, None, k, v, i32([prompt] * B), i32([prompt] + [0] * (B - 1)), None, None, c.K, c.V)
        lens, shared = i32([prompt] * B), i32([prompt] * B)
        w = torch.zeros((B, Hkv, cap), device="cuda")
        V64 = None
        a, d = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hq, 128), device="cuda")
        for t in range(own):
            qkv = torch.randn((B, 1, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).cuda()
            q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
            lens += 1
            q_rot = torch.zeros((B, 1, Hq, 128), dtype=torch.bfloat16, device="cuda")
            sfi.sfi_rope_append(ctx.handle, q, k, v, lens, None, None, q_rot, c.K, c.V)
            sfi.sfi_shared_attn(ctx.handle, q_rot.view(B, Hq, 128), c.K, c.V, lens, shared, 0, prompt, 0, a)
            sfi.sfi_weight_attn(ctx.handle, q_rot.view(B, Hq, 128), c.K, c.V, lens, 0, 1.0, w, w, d)
            torch.cuda.synchronize()
            n = prompt + t + 1
            K64, V64, q64 = to64(c.numpy(0)), to64(c.numpy(1)), to64(bits(q_rot)).reshape(B, Hq, 128)
            for b in range(B):
                o, p, size = ref.attend(q64[b], K64[b, :, :n], V64[b, :, :n])
                bound = ref.out_bound(p, V64[b, :, :n], Hq, size, o, False)
                assert (np.abs(a[b].cpu().numpy() - o) <= bound).all() and (np.abs(d[b].cpu().numpy() - o) <= bound).all(), (t, b)
        old, w_old = [c.numpy(0), c.numpy(1)], w.cpu().numpy()
        kept, n_kept = torch.zeros((B, Hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros((B, Hkv), dtype=torch.int32, device="cuda")
        sfi.sfi_evict(ctx.handle, c.K, c.V, lens, 0, budget, w, None, ctx.handle, c.K, c.V, lens, None, w, None, kept, n_kept)
        torch.cuda.synchronize()
        new = [c.numpy(0), c.numpy(1)]
        assert lens.tolist() == [prompt + budget + recent] * B
        for b in range(B):
            for h in range(Hkv):
                stay, _ = ref.kept_rows(w_old[b, h], cap, prompt, recent, budget)
                assert list(stay[:prompt]) == list(range(prompt))
                for i in (0, 1):
                    assert np.array_equal(new[i][b, h, :len(stay)], old[i][b, h, stay])
        sfi.sfi_shared_attn(ctx.handle, q_rot.view(B, Hq, 128), c.K, c.V, lens, shared, 0, prompt, 0, a)
        torch.cuda.synchronize()
        n = prompt + budget + recent
        for b in range(B):
            k, v = to64(new[0])[b, :, :n], to64(new[1])[b, :, :n]
            o, p, size = ref.attend(q64[b], k, v)
            assert (np.abs(a[b].cpu().numpy() - o) <= ref.out_bound(p, v, Hq, size, o, False)).all()
        assert sfi.sfi_device_status(ctx.handle) == 0
    finally:
        ctx.close()


def test_a_step_as_a_captured_graph():
    """Append, weighed attention and shared attention of a step captured once and replayed for steps whose lengths and positions the device holds:
    the bits of the eager calls, with eager work between the replays."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, cap, steps = 3, 8, 2, 300, 5
    g = torch.Generator().manual_seed(81)
    toks = torch.randn((steps, B, 1, Hq + 2 * Hkv, 128), generator=g).to(torch.bfloat16).cuda()
    results = []
    for replayed in (False, True):
        c = ref.Cache(B, Hkv, cap, "token", seed=80)
        ctx = c.context(Hq)
        try:
            sfi.sfi_set_rope(ctx.handle, 128)
            lens, shared = i32([200, 31, 0]), i32([0, 0, 0])
            w = torch.zeros((B, Hkv, cap), device="cuda")
            qkv, q_rot = toks[0].clone(), torch.zeros((B, 1, Hq, 128), dtype=torch.bfloat16, device="cuda")
            q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
            a, d = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hq, 128), device="cuda")

            def step():
                sfi.sfi_rope_append(ctx.handle, q, k, v, lens, None, None, q_rot, c.K, c.V)
                sfi.sfi_weight_attn(ctx.handle, q_rot.view(B, Hq, 128), c.K, c.V, lens, 0, 0.9, w, w, a)
                sfi.sfi_shared_attn(ctx.handle, q_rot.view(B, Hq, 128), c.K, c.V, lens, shared, 0, 64, 0, d)

            graph = None
            if replayed:
                s = torch.cuda.Stream()
                s.wait_stream(torch.cuda.current_stream())
                graph = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.stream(s):
                    graph.capture_begin()
                    step()
                    graph.capture_end()
                torch.cuda.current_stream().wait_stream(s)
            seen = []
            for t in range(steps):
                qkv.copy_(toks[t])
                lens += 1
                _step(f"{'replay' if replayed else 'eager'} {t}")
                graph.replay() if replayed else step()
                torch.cuda.synchronize()
                seen += [a.clone(), d.clone(), w.clone(), q_rot.clone()]
            results.append(seen + [t.clone() for t in c.store])
        finally:
            ctx.close()
    assert all(torch.equal(x, y) for x, y in zip(*results))


@pytest.mark.parametrize("layout", ["head", "htd"])
@pytest.mark.parametrize("mode", [0, 1])
def test_next_to_slow_and_fast_steps_on_one_context(layout, mode):
    """Slow, fast and ragged steps give the bits they give alone when the other operators run on their context (and workspace) in between."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hq, Hkv, rows, budget, recent = 3, 16, 4, 18000, 300, 64
    c = ref.Cache(B, Hkv, rows, layout, page=64, seed=90)
    small = ref.Cache(B, Hkv, 500, "head", seed=91)
    g = torch.Generator().manual_seed(92)
    q = torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).cuda()
    lens, shared = i32([17900, 17000, 800]), i32([600, 601, 599])
    rs = lens - recent
    is_slow = torch.tensor([1, 0, 0], dtype=torch.uint8, device="cuda")
    selector = None if mode == 0 else dict(gamma=1.0, beta=0.5, p=2.0, eta=0.1, lambda_clip=0.7, alpha_soft=0.5, alpha_cross=0.5, temp=1.0, eps=1e-8, nms_radius=8)
    results = []
    for between in (False, True):
        ctx = c.context(Hq, n_sink=4, recent=recent, budget=budget, selector=selector)
        ctx_small = small.context(Hq, n_sink=4, recent=recent, budget=budget)
        try:
            w = torch.zeros((B, Hkv, rows), device="cuda")
            o = torch.zeros((B, Hq, 128), device="cuda")
            kept, n_kept, left = torch.zeros((B, Hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros((B, Hkv), dtype=torch.int32, device="cuda"), i32([0] * B)

            def others():
                if not between:
                    return
                sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, lens, 0, 1.0, w, w, o)
                sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, lens, shared, 0, 601, 0, o)
                sfi.sfi_evict(ctx.handle, c.K, c.V, lens, 0, budget, w, None, ctx_small.handle, small.K, small.V, left, None, None, None, kept, n_kept)
                sfi.sfi_evict(ctx.handle, c.K, c.V, i32([900, 700, 800]), 1000, budget, w, None, ctx_small.handle, small.K, small.V, left, None, None, None, kept, n_kept)

            seen = []
            for _ in range(2):
                out, idx, n = (torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hkv, budget), dtype=torch.int32, device="cuda"),
                               torch.zeros((B, Hkv), dtype=torch.int32, device="cuda"))
                others()
                sfi.sfi_slow_step(ctx.handle, q, c.K, c.V, lens, 0, budget, out, idx, n)
                seen += [out.clone(), idx.clone(), n.clone()]
                others()
                sfi.sfi_fast_step(ctx.handle, q, c.K, c.V, idx, n, budget, rs, lens, out)
                seen.append(out.clone())
                others()
                sfi.sfi_mixed_step(ctx.handle, q, c.K, c.V, is_slow, lens, rs, 0, budget, out, idx, n)
                seen += [out.clone(), idx.clone(), n.clone()]
                others()
                sfi.sfi_dense_attn(ctx.handle, q, c.K, c.V, lens, 0, out)
                seen.append(out.clone())
            torch.cuda.synchronize()
            assert sfi.sfi_device_status(ctx.handle) == 0
            results.append(seen)
        finally:
            ctx.close()
            ctx_small.close()
    assert all(torch.equal(x, y) for x, y in zip(*results))


@pytest.mark.parametrize("bad_id", [-1, 1 << 30])
@pytest.mark.parametrize("B, Hq, Hkv", [(3, 4, 2), (3, 24, 2), (20, 32, 2)])
def test_block_ids_outside_the_pool(B, Hq, Hkv, bad_id):
    """One sequence's table names blocks that are not there: reported, the other sequences as they were, nothing written outside their rows."""
    import torch
    import paper_2603_12038_amd as sfi

    rows, budget, recent = 500, 60, 16
    g = torch.Generator().manual_seed(95)
    c, small = ref.Cache(B, Hkv, rows, "htd", page=16, seed=94), ref.Cache(B, Hkv, 120, "thd", page=16, seed=96)
    ctx, ctx_small = c.context(Hq, n_sink=4, recent=recent, budget=budget), small.context(Hq, n_sink=0, recent=0, budget=0)
    q = torch.randn((B, Hq, 128), generator=g).to(torch.bfloat16).cuda()
    w0 = torch.rand((B, Hkv, rows), generator=g).cuda()
    lens, shared = i32([480 - 7 * b for b in range(B)]), i32([200] * B)
    good, good_small, empty = c.table.clone(), small.table.clone(), [t.clone() for t in small.store]
    others = [b for b in range(B) if b != 1]

    def call(bad, bad_small):
        c.table.copy_(good)
        small.table.copy_(good_small)
        for t, e in zip(small.store, empty):
            t.copy_(e)
        if bad:
            c.table[1, 13:20] = bad_id
        if bad_small:
            small.table[1, 2:4] = bad_id
        a, d, w = torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hq, 128), device="cuda"), torch.zeros((B, Hkv, rows), device="cuda")
        kept, n_kept, left = torch.zeros((B, Hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros((B, Hkv), dtype=torch.int32, device="cuda"), i32([0] * B)
        seen = []
        for name in ("shared", "weigh", "evict"):
            _step(f"B={B} heads {Hq}/{Hkv} {name} bad={bad, bad_small, bad_id}")
            if name == "shared":
                sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, lens, shared, 0, 200, 0, a)
            elif name == "weigh":
                sfi.sfi_weight_attn(ctx.handle, q, c.K, c.V, lens, 0, 1.0, w0, w, d)
            else:
                sfi.sfi_evict(ctx.handle, c.K, c.V, lens, 0, budget, w0, None, ctx_small.handle, small.K, small.V, left, None, None, None, kept, n_kept)
            torch.cuda.synchronize()
            seen.append(sfi.sfi_device_status(ctx.handle))
        return seen, a, d, w, kept, n_kept, left, [t.clone() for t in small.store]

    try:
        want = call(False, False)
        assert want[0] == [0, 0, 0]
        got = call(True, False)
        assert got[0] == [8, 8, 8]
        for x, y in zip(got[1:4], want[1:4]):
            assert torch.equal(x[others], y[others])
        assert all(torch.equal(x, y) for x, y in zip(got[4:7], want[4:7]))
        mine = set(small.table_np[1].tolist())
        rest = [i for i in range(small.n_blocks) if i not in mine]
        for x, y in zip(got[7], want[7]):
            assert torch.equal(x[rest], y[rest])
        got = call(False, True)
        assert got[0] == [0, 0, 8]
        gone = small.table_np[1, 2:4].tolist()
        for x, y, e in zip(got[7], want[7], empty):
            keep = [i for i in range(small.n_blocks) if i not in gone]
            assert torch.equal(x[keep], y[keep]) and torch.equal(x[gone], e[gone])
    finally:
        ctx.close()
        ctx_small.close()


@pytest.mark.parametrize("Hq", [4, 24])
def test_a_leads_block_ids_outside_the_pool(Hq):
    """Reported only where the rows are used: sequences that share none of them are as they were."""
    import torch
    import paper_2603_12038_amd as sfi

    B, Hkv, rows = 3, 2, 400
    c = ref.Cache(B, Hkv, rows, "htd", page=16, seed=97)
    ctx = c.context(Hq)
    q = torch.randn((B, Hq, 128), generator=torch.Generator().manual_seed(98)).to(torch.bfloat16).cuda()
    lens = i32([350, 340, 330])
    try:
        out = []
        for shared, bad in (([192, 192, 0], False), ([192, 192, 0], True)):
            if bad:
                c.table[0, 3] = c.n_blocks
            o = torch.zeros((B, Hq, 128), device="cuda")
            _step(f"lead, heads {Hq}/{Hkv} bad={bad}")
            sfi.sfi_shared_attn(ctx.handle, q, c.K, c.V, lens, i32(shared), 0, 192, 0, o)
            torch.cuda.synchronize()
            assert sfi.sfi_device_status(ctx.handle) == (8 if bad else 0)
            out.append(o)
        assert torch.equal(out[0][2], out[1][2]) and out[1].isfinite().all()
    finally:
        ctx.close()
