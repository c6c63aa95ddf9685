"""The Python side of sfi_rope_append (no GPU): what it takes, what it refuses, and the strides that reach the library."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

import paper_2603_12038_amd as sfi
from paper_2603_12038_amd import binding
from test_boundary import good_cfg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class _Recorder:
    def sfi_rope_append(self, ctx, q, qb, qt, k, kb, kt, v, vb, vt, *rest):
        self.strides, self.new = (qb, qt, kb, kt, vb, vt), rest[3]


@pytest.fixture()
def recorder(monkeypatch):
    r = _Recorder()
    monkeypatch.setattr(binding, "_hot", r)
    return r


@pytest.fixture()
def handle():
    """A context of 2 sequences, 8 query heads, 2 KV heads (never run: there is no memory behind it)."""
    cfg = good_cfg(batch=2, n_q_heads=8, n_kv_heads=2)
    h = sfi.sfi_create(cfg, 0x10000, sfi.sfi_workspace_bytes(cfg))
    yield h
    sfi.sfi_destroy(h)


def _rows(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _call(ctx, **over):
    a = dict(q=_rows(2, 3, 8, 128), k=_rows(2, 3, 2, 128), v=_rows(2, 3, 2, 128), q_out=_rows(2, 3, 8, 128))
    a.update(over)
    sfi.sfi_rope_append(ctx, a["q"], a["k"], a["v"], None, None, None, a["q_out"], 0x20000, 0x20000, stream=1)


def test_strides_of_a_projections_parts(recorder, handle):
    qkv = _rows(2, 3, 12, 128)
    q, k, v = qkv.split([8, 2, 2], dim=2)
    _call(handle, q=q, k=k, v=v)
    assert recorder.strides == (3 * 1536, 1536) * 3 and recorder.new == 3
    _call(C.c_void_p(handle), q=None, q_out=None)
    assert recorder.strides == (0, 0, 768, 256, 768, 256)


def test_strides_of_dimensions_of_one_are_not_passed_on(recorder, handle):
    """torch may give a dimension of one any stride, an odd one too."""
    odd = lambda heads: _rows(4096).as_strided((2, 1, heads, 128), (heads * 128, 5, 128, 1))  # noqa: E731
    _call(handle, q=odd(8), k=odd(2), v=odd(2), q_out=_rows(2, 1, 8, 128))
    assert recorder.strides == (1024, 0, 256, 0, 256, 0)
    cfg = good_cfg(batch=1, n_q_heads=1, n_kv_heads=1)
    h = sfi.sfi_create(cfg, 0x10000, sfi.sfi_workspace_bytes(cfg))
    try:
        one = _rows(4096).as_strided((1, 3, 1, 128), (3, 136, 7, 1))
        _call(h, q=one, k=one, v=one, q_out=_rows(1, 3, 1, 128))
        assert recorder.strides == (0, 136) * 3
    finally:
        sfi.sfi_destroy(h)


@pytest.mark.parametrize("over", [
    dict(k=_rows(2, 3, 2, 64), v=_rows(2, 3, 2, 64)),  # not 128 elements a head
    dict(k=_rows(2, 3, 2, 128)[..., :64], v=_rows(2, 3, 2, 128)[..., :64]),  # nor where the heads lie 128 apart
    dict(k=_rows(2, 3, 4, 128), v=_rows(2, 3, 4, 128)), dict(v=_rows(2, 3, 4, 128)), dict(v=_rows(2, 2, 2, 128)),  # other heads, other rows
    dict(q=_rows(2, 3, 2, 128), q_out=_rows(2, 3, 2, 128)), dict(q=_rows(2, 4, 8, 128)), dict(q=_rows(1, 3, 8, 128)),
    dict(q_out=_rows(2, 3, 4, 128)), dict(q_out=_rows(2, 2, 8, 128)), dict(q_out=_rows(3, 2, 8, 128).transpose(0, 1)),
    dict(k=_rows(1, 3, 2, 128), v=_rows(1, 3, 2, 128), q=_rows(1, 3, 8, 128), q_out=_rows(1, 3, 8, 128)),  # sequences of another context
    dict(k=_rows(2, 2, 3, 128).transpose(1, 2)), dict(v=_rows(2, 3, 2, 256)[..., ::2]), dict(q=_rows(2, 3, 16, 128)[:, :, ::2]),
    dict(k=_rows(2, 3, 256)),
])
def test_other_shapes_are_refused(recorder, handle, over):
    with pytest.raises(AssertionError):
        _call(handle, **over)
    assert not hasattr(recorder, "strides"), "the call went on to the library"


def test_refused_without_assert_statements_too():
    code = ("import torch, paper_2603_12038_amd as sfi\n"
            "k = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16)\n"
            "try:\n    sfi.sfi_rope_append(0, None, k, k, None, None, None, None, 64, 64, stream=1)\n"
            "except AssertionError as e:\n    print('refused', e)\n")
    r = subprocess.run([sys.executable, "-O", "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.startswith("refused k: "), r.stderr


def test_a_handle_is_forgotten_with_its_context(recorder):
    cfg = good_cfg(batch=2, n_q_heads=8, n_kv_heads=2)
    h = sfi.sfi_create(cfg, 0x10000, sfi.sfi_workspace_bytes(cfg))
    assert binding._heads[h] == (2, 8, 2)
    sfi.sfi_destroy(C.c_void_p(h))
    assert h not in binding._heads


