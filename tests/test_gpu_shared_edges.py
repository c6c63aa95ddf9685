"""sfi_shared_attn where it could answer wrongly without a word: what is no number stays none, weights keep their bits, bounds that are loose."""
import numpy as np
import pytest

import cache_ref as ref
from cache_ref import bits, i32, to64

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
