"""Plain 64-bit forms of the calls on rows of logits, and bounds on what 32-bit arithmetic may differ from them by.

Bounds.  u = 2^-24.  Of y = scale (z - m) the difference and the product are rounded: |error| <= 2 u |y|, one more u |y| for the
factor log2(e) and 2^-22 for the power of two, so a term e = exp(y) is off by (2^-22 + 3 u |y|) e, and the sum of V terms, of which at
least 128 partial sums are formed side by side, by another (V / 128 + 64) u s.  With the averages Y = sum e |y| / s and Y2 = sum e y^2 / s:
  log s      2^-22 + 3 u Y + (V / 128 + 64) u, and u |log s| for the logarithm itself (2 ulp: 4 u)
  log p      that, and 4 u (|y| + |log s|) for y and the subtraction
  entropy    twice the first, (2^-22 + chain) Y + 3 u Y2 for the sum of e y, 4 u H for the last operations
  p          p times (log p's bound + 2^-22 + 2 u |log p|)
A result rounded to bf16 is off by another 2^-9 of itself (and by half of the smallest positive value).
"""
import ctypes as C

import numpy as np
import torch

from paper_2204_04179_b200 import binding

DEV = "cuda:0"
U = 2.0 ** -24
INF = np.inf
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def context():
    cfg = binding.GramConfig()
    cfg.n_items, cfg.P_max, cfg.d = 1, 1, 8
    return binding.Gram(cfg)


def buffer(N, V, dtype, pad=0, offset=0, fill=float("nan")):
    """An [N, V] view with rows V + pad elements apart that begins `offset` elements into its allocation; NaN around it."""
    flat = torch.full((offset + N * (V + pad) + 8,), fill, dtype=DT[dtype], device=DEV)
    return flat, flat[offset:].as_strided((N, V), (V + pad, 1))


def place(z, dtype, pad=0, offset=0):
    """The rows z (float64 numpy) on the device, and their values as the device holds them."""
    flat, view = buffer(z.shape[0], z.shape[1], dtype, pad, offset)
    view.copy_(torch.from_numpy(z).to(DT[dtype]))
    return view, view.double().cpu().numpy()


class Rows:
    """Softmax of rows of logits in 64 bits, with the bounds above."""

    def __init__(self, z, scale):
        with np.errstate(all="ignore"):
            self.z, self.scale = z, float(np.float32(scale))
            self.V = z.shape[1]
            m = z.max(1)
            self.m = m
            self.y = self.scale * (z - np.where(np.isneginf(m), 0.0, m)[:, None])
            e = np.exp(self.y)
            s = e.sum(1)
            self.s, self.log_s = s, np.log(s)
            self.empty = s == 0
            ls = np.where(self.empty, 0.0, self.log_s)
            self.p = np.where(self.empty[:, None], 0.0, e / np.where(self.empty, 1.0, s)[:, None])
            self.logp = np.where(np.isneginf(z), -INF, self.y - ls[:, None])
            yy = np.where(e > 0, self.y, 0.0)
            self.H = np.where(self.empty, 0.0, ls - (self.p * yy).sum(1))
            Y, Y2 = (self.p * np.abs(yy)).sum(1), (self.p * yy ** 2).sum(1)
            chain = (self.V / 128 + 64) * U
            self.d_log_s = 2.0 ** -22 + 3 * U * Y + chain + 4 * U * np.abs(ls)
            self.d_H = 2 * self.d_log_s + (2.0 ** -22 + chain) * Y + 3 * U * Y2 + 4 * U * self.H
            self.d_logp = self.d_log_s[:, None] + 4 * U * (np.abs(np.where(np.isinf(self.y), 0, self.y)) + np.abs(ls)[:, None])
            self.d_p = self.p * (self.d_logp + 2.0 ** -22 + 2 * U * np.abs(np.where(np.isinf(self.logp), 0, self.logp)))

    def top(self, k):
        ids = np.full((self.z.shape[0], k), -1, np.int32)
        for n, row in enumerate(self.z):
            order = [v for v in np.lexsort((np.arange(self.V), -row)) if row[v] > -INF][:k]
            ids[n, :len(order)] = order
        return ids

    def at(self, table, ids, none):
        got = np.take_along_axis(table, np.maximum(ids, 0).astype(np.int64), 1)
        return np.where(ids >= 0, got, none)


def near(got, want, bound, what):
    """Equal where infinite, else within the bound."""
    got = got.double().cpu().numpy() if torch.is_tensor(got) else np.asarray(got, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), what
    off = np.abs(got - want)[fine] - np.broadcast_to(bound, want.shape)[fine]
    assert got.shape == want.shape and np.isfinite(got[fine]).all() and (off <= 0).all(), (what, float(off.max()))


def answers(N, C=0, k=0):
    f = dict(device=DEV, dtype=torch.float32)
    nan = float("nan")
    return dict(stats=torch.full((N, 2), nan, **f), entropy=torch.full((N,), nan, **f), logp=torch.full((N, C), nan, **f) if C else None,
                top_logp=torch.full((N, k), nan, **f) if k else None,
                top_ids=torch.full((N, k), -7, device=DEV, dtype=torch.int32) if k else None)


def check_answers(out, r, targets, k, dz=0.0):
    """dz: bound on the logits themselves (products), beside which alternatives are not compared."""
    more = r.scale * dz
    near(out["stats"][:, 0], r.m, np.where(np.isfinite(r.m), dz, 0.0), "m")
    near(out["stats"][:, 1], r.log_s, r.d_log_s + 2 * more, "log s")
    Y = np.abs(np.where(r.p > 0, r.y, 0)).max(1)
    near(out["entropy"], r.H, r.d_H + 4 * more * (1 + Y), "entropy")
    if targets is not None:
        near(out["logp"], r.at(r.logp, targets, 0.0), r.at(r.d_logp, targets, 0.0) + 4 * more, "log p")
    if k:
        ids = r.top(k)
        assert np.array_equal(out["top_ids"].cpu().numpy(), ids)
        near(out["top_logp"], r.at(r.logp, ids, -INF), r.at(r.d_logp, ids, 0.0) + 4 * more, "log p of alternatives")
