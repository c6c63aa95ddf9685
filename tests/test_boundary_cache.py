"""What sfi_set_rope, sfi_rope_append, sfi_shared_attn, sfi_weight_attn and sfi_evict refuse on the host, before anything is launched (no GPU),
and the angles of the rotary rules."""
import ctypes as C
import math

import numpy as np
import pytest

import cache_ref as ref
import paper_2603_12038_amd as sfi
from paper_2603_12038_amd.binding import SfiRope
from test_boundary import EALIGN, EINVAL, EUNSUPPORTED, OK, good_cfg

P = 0x20000  # stands for any 16-byte aligned device pointer; never used by a failing call


@pytest.fixture()
def ctx():
    lib = sfi.load_library()
    made = []

    def make(**over):
        cfg = good_cfg(**over)
        h = C.c_void_p()
        assert lib.sfi_create(C.byref(cfg), 0x10000, sfi.sfi_workspace_bytes(cfg), C.byref(h)) == OK
        made.append(h)
        return h

    yield make
    for h in made:
        lib.sfi_destroy(h)


PAGED = dict(page_size=16, k_stride_b=0, v_stride_b=0, k_stride_t=256, k_stride_h=128, v_stride_t=256, v_stride_h=128)


# ---- rotary rules ----

@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
@pytest.mark.parametrize("scaling", [None, dict(kind="linear", factor=4.0), dict(kind="turns", factor=8.0, low=1.0, high=4.0, orig_ctx=8192),
                                     dict(kind="dims", factor=40.0, low=1.0, high=32.0, orig_ctx=4096), dict(kind="dims", factor=2.0, low=0.5, high=0.75, orig_ctx=1)])
def test_angles_of_the_rules(rot, base, scaling):
    got, want = np.array(sfi.sfi_rope_freqs(rot, base, scaling)), np.array(ref.freqs(rot, base, scaling))
    # the same few operations in 64 bits; the ramp multiplies what two divisions and a logarithm round
    assert got.shape == (rot // 2,) and np.allclose(got, want, rtol=64 * 2.0 ** -53, atol=0)


def test_a_rule_leaves_fast_pairs_and_stretches_slow_ones():
    for kind in ("turns", "dims"):
        f = sfi.sfi_rope_freqs(128, 500000.0, dict(kind=kind, factor=8.0, low=1.0, high=4.0, orig_ctx=8192))
        w = sfi.sfi_rope_freqs(128, 500000.0)
        assert f[0] == w[0] and math.isclose(f[-1], w[-1] / 8) and all(a / 8 <= b * (1 + 1e-15) and b <= a for a, b in zip(w, f))


def _rope(**over):
    r = SfiRope()
    r.rot_dim, r.base, r.factor, r.low, r.high, r.orig_ctx = 128, 10000.0, 2.0, 1.0, 4.0, 4096
    for k, v in over.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("over, code", [
    (dict(rot_dim=0), EINVAL), (dict(rot_dim=-16), EINVAL), (dict(rot_dim=144), EINVAL), (dict(rot_dim=40), EUNSUPPORTED), (dict(rot_dim=15), EUNSUPPORTED),
    (dict(interleaved=2), EINVAL), (dict(base=1.0), EINVAL), (dict(base=float("nan")), EINVAL), (dict(base=float("inf")), EINVAL),
    (dict(scaling=4), EUNSUPPORTED), (dict(scaling=-1), EUNSUPPORTED), (dict(scaling=1, factor=0.0), EINVAL), (dict(scaling=1, factor=float("nan")), EINVAL),
    (dict(scaling=2, low=4.0), EINVAL), (dict(scaling=2, orig_ctx=0), EINVAL), (dict(scaling=3, low=0.0), EINVAL), (dict(scaling=3, high=float("inf")), EINVAL),
    (dict(magnitude=-1.0), EINVAL), (dict(magnitude=float("nan")), EINVAL),
])
def test_rules_that_are_refused(ctx, over, code):
    lib, f = sfi.load_library(), (C.c_double * 64)()
    assert lib.sfi_rope_freqs(C.byref(_rope(**over)), f) == code
    assert lib.sfi_set_rope(ctx(), C.byref(_rope(**over)), None) == code


def test_rope_arguments(ctx):
    lib, f = sfi.load_library(), (C.c_double * 64)()
    assert lib.sfi_rope_freqs(C.byref(_rope()), f) == OK
    assert lib.sfi_rope_freqs(None, f) == EINVAL and lib.sfi_rope_freqs(C.byref(_rope()), None) == EINVAL
    assert lib.sfi_set_rope(None, C.byref(_rope()), None) == EINVAL and lib.sfi_set_rope(ctx(), None, None) == EINVAL
    given = (C.c_double * 64)(*[0.5] * 63, float("inf"))
    assert lib.sfi_rope_freqs(C.byref(_rope(freqs=given)), f) == EINVAL
    given[63] = 0.25
    assert lib.sfi_rope_freqs(C.byref(_rope(freqs=given, base=0.0)), f) == OK and f[63] == 0.25
    assert lib.sfi_rope_freqs(C.byref(_rope(freqs=given, scaling=1)), f) == EINVAL  # given angles are not scaled
    for bad in (dict(kind="turns", factor=2.0), dict(kind="linear", factor=2.0, low=1.0)):
        with pytest.raises(ValueError):
            sfi.sfi_rope_freqs(64, 10000.0, bad)
    with pytest.raises(KeyError):
        sfi.sfi_rope_freqs(64, 10000.0, dict(kind="none", factor=1.0, low=1.0, high=2.0, orig_ctx=1))
    with pytest.raises(ValueError):
        sfi.sfi_set_rope(ctx(), 64, freqs=[0.1] * 31, stream=1)


# ---- calls ----

def _append(h, **over):
    a = dict(q=P, qb=1024, qt=1024, k=P, kb=256, kt=256, v=P, vb=256, vt=256, ctx_len=P, n_new=None, pos=None, max_new=1, q_out=P, K=P, V=P)
    assert set(over) <= set(a)
    return sfi.load_library().sfi_rope_append(h, *{**a, **over}.values(), None)


def test_append_refuses(ctx):
    assert _append(None) == EINVAL
    assert _append(ctx()) == EINVAL  # no rule yet
    assert _append(ctx(**PAGED)) == EINVAL
    # (with a rule: a context can only be given one where there is a device, so the checks behind that one run in the GPU tests too)


def test_more_rows_than_a_launch_takes(ctx):
    many = ctx(batch=1 << 15, max_ctx=4096)
    assert _append(many, max_new=4096) == EUNSUPPORTED  # 2^27 rows
    assert _append(many, max_new=0) == EINVAL and _append(many, max_new=4097) == EINVAL


@pytest.mark.parametrize("factor", [0.0, 1e-300, 9e-10, 2e9, float("inf")])
@pytest.mark.parametrize("scaling", [1, 2, 3])
def test_factors_that_leave_no_angle(factor, scaling):
    assert sfi.load_library().sfi_rope_freqs(C.byref(_rope(scaling=scaling, factor=factor)), (C.c_double * 64)()) == EINVAL


def _rows(name, h, **over):
    lib = sfi.load_library()
    a = (dict(q=P, K=P, V=P, ctx_len=P, shared_len=P, lead=0, max_shared=64, max_len=0, out=P) if name == "sfi_shared_attn" else
         dict(q=P, K=P, V=P, ctx_len=P, max_len=0, decay=1.0, weights=P, weights_out=P, out=P))
    assert set(over) <= set(a)
    return getattr(lib, name)(h, *{**a, **over}.values(), None)


@pytest.mark.parametrize("over, code", [
    (dict(q=None), EINVAL), (dict(K=None), EINVAL), (dict(V=None), EINVAL), (dict(ctx_len=None), EINVAL), (dict(shared_len=None), EINVAL),
    (dict(out=None), EINVAL), (dict(lead=-1), EINVAL), (dict(lead=2), EINVAL), (dict(max_shared=-1), EINVAL), (dict(max_shared=4097), EINVAL),
    (dict(max_shared=65, max_len=64), EINVAL), (dict(max_len=4097), EINVAL), (dict(max_len=-1), EINVAL),
    (dict(q=P + 2), EALIGN), (dict(K=P + 8), EALIGN), (dict(out=P + 4), EALIGN), (dict(shared_len=P + 2), EALIGN), (dict(ctx_len=P + 1), EALIGN),
])
def test_shared_attention_refuses(ctx, over, code):
    assert _rows("sfi_shared_attn", ctx(), **over) == code


@pytest.mark.parametrize("over, code", [
    (dict(q=None), EINVAL), (dict(V=None), EINVAL), (dict(weights_out=None), EINVAL), (dict(decay=-0.1), EINVAL), (dict(decay=1.1), EINVAL),
    (dict(decay=float("nan")), EINVAL), (dict(max_len=4097), EINVAL), (dict(weights=P + 2), EALIGN), (dict(weights_out=P + 1), EALIGN), (dict(V=P + 4), EALIGN),
])
def test_weighing_attention_refuses(ctx, over, code):
    assert _rows("sfi_weight_attn", ctx(), **over) == code


@pytest.mark.parametrize("name", ["sfi_shared_attn", "sfi_weight_attn"])
def test_no_context_or_no_block_table(ctx, name):
    assert _rows(name, None) == EINVAL
    assert _rows(name, ctx(**PAGED)) == EINVAL


def test_shared_attention_takes_four_rows_within_32_bits(ctx):
    lib = sfi.load_library()
    for over in (dict(k_stride_t=1 << 29), dict(v_stride_t=1 << 29)):
        h = ctx(**{**PAGED, **over})
        assert lib.sfi_set_block_table(h, P, 256, 4) == OK
        assert _rows("sfi_shared_attn", h) == EUNSUPPORTED


def _evict(h, to, **over):
    a = dict(K=P, V=P, ctx_len=P, max_len=0, budget=64, weights=P, row_pos=P, dst=to, K_out=2 * P, V_out=2 * P, ctx_len_out=P, recent_start_out=P,
             weights_out=2 * P, row_pos_out=2 * P, kept=P, n_kept=P)
    assert set(over) <= set(a)
    return sfi.load_library().sfi_evict(h, *{**a, **over}.values(), None)


@pytest.mark.parametrize("over, code", [
    *[({k: None}, EINVAL) for k in ("K", "V", "ctx_len", "weights", "dst", "K_out", "V_out", "ctx_len_out", "kept", "n_kept", "row_pos")],
    *[({k: P + 2}, EALIGN) for k in ("K", "V_out", "ctx_len", "weights", "row_pos", "recent_start_out", "weights_out", "row_pos_out", "kept", "n_kept")],
    (dict(K_out=2 * P + 8), EALIGN), (dict(budget=-1), EINVAL), (dict(budget=257), EINVAL), (dict(max_len=-1), EINVAL), (dict(max_len=4097), EINVAL),
    (dict(K_out=P), EINVAL), (dict(V_out=P), EINVAL),  # in place means both
])
def test_evict_refuses(ctx, over, code):
    h = ctx()
    assert _evict(h, ctx(), **over) == code


def test_evict_refuses_a_target_that_does_not_fit(ctx):
    h = ctx()
    assert _evict(None, h) == EINVAL
    assert _evict(h, ctx(batch=3)) == EINVAL and _evict(h, ctx(n_kv_heads=4)) == EINVAL
    assert _evict(h, ctx(max_ctx=4 + 64 + 64 - 1)) == EINVAL  # a row less than can be left
    assert _evict(h, ctx(**PAGED)) == EINVAL and _evict(ctx(**PAGED), h) == EINVAL  # no block table
    for over in (dict(k_stride_t=256), dict(v_stride_h=128 * 8192), dict(k_stride_b=0)):  # in place, laid out otherwise
        assert _evict(h, ctx(**over), K_out=P, V_out=P) == EINVAL
    small = ctx(max_ctx=2048)
    assert _evict(h, small, weights_out=P) == EINVAL and _evict(h, small, row_pos_out=P) == EINVAL  # one array cannot have two lengths


def test_python_names_and_shapes():
    import torch

    k = torch.zeros((2, 3, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        sfi.sfi_rope_append(0, None, k, k.transpose(1, 2), None, None, None, None, k, k)
    with pytest.raises(AssertionError):
        sfi.sfi_rope_append(0, None, k, k[..., ::2], None, None, None, None, k, k)
    with pytest.raises(sfi.SfiError) as e:
        sfi.sfi_rope_append(0, None, k, k, None, None, None, None, k, k, stream=1)
    assert e.value.code == EINVAL
    with pytest.raises(TypeError):
        sfi.sfi_weight_attn(0, k, k, k, k, 0, "1", None, k, k, stream=1)
