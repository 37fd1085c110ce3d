"""Plain models in 64 bits of what an 8-bit pool holds and computes, written from the definitions in include/ekv.h;
they share nothing with the library."""
import numpy as np
import torch

E_LO, E_HI = -112, 120


def _code_values():
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if (c & 127) == 127 else (-x if c & 128 else x)
    return v


CODE_VALUE = _code_values()                 # 256 values, NaN at 0x7f and 0xff
_MAG = CODE_VALUE[:127]                     # ascending magnitudes of codes 0 .. 0x7e


def encode(x):
    """float64 -> codes: the nearest value, ties to the even code; NaN -> 0x7f (with its sign dropped)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_MAG, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = _MAG[hi] - a, a - _MAG[lo]
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(hi % 2 == 0, hi, lo)))
    pick = np.where(np.isnan(x), 127, pick).astype(np.uint8)
    return np.where(np.signbit(x) & ~np.isnan(x), pick | 128, pick).astype(np.uint8)


def scale_of(a):
    """The smallest 2^e, e in [E_LO, E_HI], with a <= 448 * 2^e."""
    e = E_LO
    if a > 0:
        e = max(E_LO, int(np.frexp(a)[1]) - 11)
        while e < E_HI and a > 448 * 2.0 ** e:
            e += 1
    return 2.0 ** min(e, E_HI)


class Cache:
    """codes uint8 [blocks, 2, Hk, 16, D] and scales float64 [blocks, 2, Hk]."""

    def __init__(self, blocks, Hk, D, fill=0x7F):
        self.codes = np.full((blocks, 2, Hk, 16, D), fill, dtype=np.uint8)
        self.scales = np.zeros((blocks, 2, Hk))

    def write(self, k, v, slots):
        """k, v: float64 [T, Hk, D].  Returns whether some slot was out of range."""
        rows, oob = {}, False
        for t, s in enumerate(np.asarray(slots)):
            if s < 0:
                continue
            if s // 16 >= len(self.codes):
                oob = True
                continue
            rows.setdefault(int(s // 16), {})[int(s % 16)] = t          # the last of duplicates stays
        for n, of in rows.items():
            # a duplicate that loses does not reach the cache, nor the maximum
            for kv, x in enumerate((k, v)):
                for h in range(x.shape[1]):
                    new = np.stack([x[t, h] for t in of.values()])
                    fin = np.abs(new[np.isfinite(new)])
                    old = 0.0 if 0 in of else self.scales[n, kv, h]
                    s = max(old, scale_of(fin.max() if fin.size else 0.0))
                    for o in range(16):
                        if o in of:
                            y = np.where(np.isfinite(x[of[o], h]), x[of[o], h], np.nan) / s
                            if s == 2.0 ** E_HI:
                                y = np.clip(y, -240, 240)
                            self.codes[n, kv, h, o] = encode(y)
                        elif 0 < old < s:
                            self.codes[n, kv, h, o] = encode(CODE_VALUE[self.codes[n, kv, h, o]] * (old / s))
                    self.scales[n, kv, h] = s
        return oob

    def values(self):
        return CODE_VALUE[self.codes] * self.scales[..., None, None]

    def rows(self, slots):
        """(k, v) float64 [T, Hk, D] of valid slots; a tile that was never written is 0."""
        slots = np.asarray(slots)
        scales = self.scales[slots // 16][..., None]
        x = np.where(scales > 0, CODE_VALUE[self.codes[slots // 16, :, :, slots % 16]] * scales, 0.0)
        return x[:, 0], x[:, 1]


def attention(q, K, V, limits, scale, sv=None):
    """q [c, Hq, D], K and V [L, Hk, D] float64; row i sees keys j < limits[i] with `valid` rows (NaN rows of K stand for keys
    that are skipped).  sv: V's scale of each key and head [L, Hk], for the bound.  Returns (out, bound): bound is how far a bf16 result may be off (see below)."""
    q, K, V = (torch.as_tensor(x, dtype=torch.float64) for x in (q, K, V))
    c, Hq, D = q.shape
    L, Hk, _ = K.shape
    G = Hq // Hk
    out, bound = torch.zeros(c, Hq, D, dtype=torch.float64), torch.zeros(c, Hq, D, dtype=torch.float64)
    if L == 0:
        return out, bound
    skip = torch.isnan(K[:, 0, 0])
    seen = (torch.arange(L) < torch.as_tensor(limits)[:, None]) & ~skip
    K, V = torch.nan_to_num(K), torch.where(skip[:, None, None], torch.zeros(()).double(), V)
    for h in range(Hq):
        s = q[:, h] @ K[:, h // G].T * scale
        s = torch.where(seen, s, torch.full((), -torch.inf, dtype=torch.float64))
        m = s.amax(1, keepdim=True)
        p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
        l = p.sum(1, keepdim=True)
        p = p / torch.where(l > 0, l, torch.ones_like(l))
        out[:, h] = p @ V[:, h // G]
        # Derivation.  P is rounded to bf16 (half a step: 2^-8 of it), the sum is exact to fp32, and the result is rounded to
        # bf16 (2^-8): 2^-8 (sum p |v| + |out|).  Scores are fp32 sums of D products, each step and the scaling within 2^-23 of the
        # sum of magnitudes, and exp2 is within 2^-21: a relative error d of every weight moves the quotient by at most
        # 2 d sum p |v|.  Zero results aside, an fp32 sum of L weights adds (L + 200) 2^-24 of sum p |v|.
        size = p @ V[:, h // G].abs()
        reach = (q[:, h].abs() @ K[:, h // G].abs().T * abs(scale)).where(seen, torch.zeros(()).double()).amax(1, keepdim=True)
        d = (D + 4) * 2.0 ** -23 * reach + 2.0 ** -21
        # P in f16 (decode, few rows): 2^-11 of it, less than the above, down to 2^-14, and half of f16's smallest step, 2^-25, below.
        # P is exp2 of the score with V's exponent on top, scaled so that a row's largest is 2^6 at least: 2^-31 of the largest
        # p_j s_j at most for each key, times its code, which is 448 at most.
        floor = 0.0 if sv is None else 2.0 ** -31 * 448 * seen.sum(1, keepdim=True) * (p * torch.as_tensor(sv, dtype=torch.float64)[:, h // G]).amax(1, keepdim=True)
        bound[:, h] = floor + 2.0 ** -8 * (size + out[:, h].abs()) + (2 * d + (L + 200) * 2.0 ** -24) * size + 1e-30
    return out, bound


def assert_within(got, want, bound, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (got.shape, want.shape)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, worst ratio {float(((got - want).abs() / bound).nan_to_num(1e9).max()):.3g}"
