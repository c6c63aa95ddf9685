"""Plain 64-bit forms (numpy, CPU) of what stands around the decode step, and caches of every layout to run it on."""
import math

import numpy as np
import torch

D = 128


# ---- caches ----------------------------------------------------------------------------------------------------------

class Cache:
    """K and V of `rows` rows for B sequences on the GPU.  layout: "head" [B, Hkv, rows, 128]; "token" the same from [B, rows, Hkv, 128];
    "wide" rows 136 apart; "htd" / "thd" pools of blocks of `page` rows behind a shuffled block table, with spare blocks."""

    def __init__(self, B, Hkv, rows, layout, page=16, seed=0, fill="normal", device="cuda"):
        self.B, self.Hkv, self.rows, self.layout = B, Hkv, rows, layout
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.paged = layout in ("htd", "thd")
        if self.paged:
            self.page = page
            per = (rows + page - 1) // page
            self.n_blocks = B * per + 3
            self.table_np = rng.permutation(self.n_blocks)[:B * per].reshape(B, per).astype(np.int32)
            shape = (self.n_blocks, Hkv, page, D) if layout == "htd" else (self.n_blocks, page, Hkv, D)
        else:
            self.page = 0
            shape = {"head": (B, Hkv, rows, D), "token": (B, rows, Hkv, D), "wide": (B, Hkv, rows, D + 8)}[layout]
        self.store = []
        for _ in range(2):
            t = torch.full(shape, float("nan"), dtype=torch.bfloat16) if fill == "nan" else torch.randn(shape, generator=g).to(torch.bfloat16)
            self.store.append(t.to(device))
        self.K, self.V = (self._view(t) for t in self.store)
        self.table = torch.from_numpy(self.table_np).to(device) if self.paged else None

    def _view(self, t):
        return t.transpose(1, 2) if self.layout == "token" else t[..., :D] if self.layout == "wide" else t

    def numpy(self, which):
        """[B, Hkv, rows, 128] of the cache's present content as bf16 bits."""
        t = (self.K, self.V)[which].contiguous().cpu().view(torch.int16).numpy().view(np.uint16)
        if not self.paged:
            return t.copy()
        if self.layout == "thd":
            t = t.transpose(0, 2, 1, 3)
        return t[self.table_np].transpose(0, 2, 1, 3, 4).reshape(self.B, self.Hkv, -1, D)[:, :, :self.rows].copy()

    def put(self, which, b, row, bits):
        """Row `row` of sequence b := bits [Hkv, 128] (uint16)."""
        v = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).to(self.K.device)
        t = (self.K, self.V)[which]
        if not self.paged:
            t[b, :, row] = v
        elif self.layout == "htd":
            t[int(self.table_np[b, row // self.page]), :, row % self.page] = v
        else:
            t[int(self.table_np[b, row // self.page]), row % self.page] = v

    def context(self, Hq, n_sink=4, recent=64, budget=256, **more):
        import paper_2603_12038_amd as sfi

        ctx = sfi.SfiContext(self.B, Hq, self.Hkv, self.rows, budget, n_sink, recent, self.K, self.V, page_size=self.page,
                             page_layout=self.layout if self.paged else "thd", **more)
        if self.paged:
            sfi.sfi_set_block_table(ctx.handle, self.table, self.n_blocks)
        return ctx


LAYOUTS = ["head", "token", "wide", "htd", "thd"]


def bits(t):
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16)


def to64(b):
    return (np.ascontiguousarray(b, dtype=np.uint16).astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


def i32(a, device="cuda"):
    return torch.tensor(np.asarray(a, np.int32), device=device)


# ---- rotary positions ------------------------------------------------------------------------------------------------

def freqs(rot, base, scaling=None):
    w = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling is None:
        return w
    kind, factor = scaling["kind"], scaling["factor"]
    if kind == "linear":
        return [x / factor for x in w]
    out = []
    for i, x in enumerate(w):
        if kind == "turns":
            s = (scaling["orig_ctx"] * x / (2 * math.pi) - scaling["low"]) / (scaling["high"] - scaling["low"])
        else:
            at = lambda n: rot * math.log(scaling["orig_ctx"] / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(math.floor(at(scaling["high"])), 0), min(math.ceil(at(scaling["low"])), rot - 1)
            s = 1 - (i - lo) / max(hi - lo, 0.001)
        s = min(1.0, max(0.0, s))
        out.append(x * (s + (1 - s) / factor))
    return out


def rotate(x, pos, f, interleaved, magnitude):
    """x: [..., heads, 128] in 64 bits at positions pos[...]; also what the terms of each output add up to in size."""
    rot = 2 * len(f)
    turn = np.longdouble("6.283185307179586476925286766559")
    angle = np.asarray(pos, np.longdouble)[..., None] * np.asarray(f, np.longdouble)  # (64 bits do not hold a far position's fraction of a turn)
    angle = (angle - np.round(angle / turn) * turn).astype(np.float64)
    c, s = magnitude * np.cos(angle)[..., None, :], magnitude * np.sin(angle)[..., None, :]
    out, size = x.copy(), np.abs(x)
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i], x[..., j]
    out[..., i], out[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = magnitude * (np.abs(a) + np.abs(b))
    return out, size


# ---- attention -------------------------------------------------------------------------------------------------------

def attend(q, K, V, scale=None):
    """q [Hq, 128], K, V [Hkv, n, 128] in 64 bits -> out [Hq, 128], softmax [Hq, n], and how large |q||k| * scale gets."""
    Hq, (Hkv, n, _) = q.shape[0], K.shape
    g = Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    if n == 0:
        return np.zeros((Hq, D)), np.zeros((Hq, 0)), 0.0
    qg = q.reshape(Hkv, g, D)
    y = np.matmul(qg, K.transpose(0, 2, 1)) * scale
    p = np.exp(y - y.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    size = float((np.matmul(np.abs(qg), np.abs(K).transpose(0, 2, 1)) * scale).max())
    return np.matmul(p, V).reshape(Hq, D), p.reshape(Hq, n), size


# fp32 sums of 128 exact products are off by at most 128 half steps (2^-24 each) of the sum of the products' sizes; so is a logit, by
# 2^-23 of itself more for the scale and the change to base 2.  A weight is off by that, by 2^-22 for the exponential, and by 2^-17 for its two bf16 terms;
# sums over rows, in any order and with rescaled parts, add less than 2^-16 at the lengths here (tree of lanes, waves, splits).
def weight_slack(size):
    return 2.0 ** -17 + 2.0 ** -16 + 2.0 ** -22 + 130 * 2.0 ** -24 * size


def out_bound(p, V, Hq, size, ref, bf16):
    """|error| allowed: every weight off by the slack, the norm too, of sum p |v|; a bf16 output rounds once more."""
    Hkv = V.shape[0]
    if V.shape[1] == 0:
        return np.zeros((Hq, D))
    mass = np.matmul(p.reshape(Hkv, Hq // Hkv, -1), np.abs(V)).reshape(Hq, D)
    b = 2 * weight_slack(size) * mass + 1e-30
    return b + (np.abs(ref) + b) * 2.0 ** -8 if bf16 else b


# ---- eviction --------------------------------------------------------------------------------------------------------

def kept_rows(w, L, n_sink, recent, budget):
    """Rows of one (sequence, KV head) that stay, ascending, and those of J among them."""
    lo, hi = n_sink, L - recent
    J = np.arange(lo, hi) if hi > lo else np.arange(0)
    key = w[J].astype(np.float32)
    key = np.where(key > 0, key, np.float32(0))
    order = sorted(range(len(J)), key=lambda i: (-key[i], i))[:budget]
    middle = J[sorted(order)].astype(np.int64)
    gone = set(J.tolist()) - set(middle.tolist())
    return np.array([r for r in range(L) if r not in gone], np.int64), middle
