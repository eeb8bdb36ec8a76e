"""Inputs of the paged entries' GPU tests: small sweeps over pools of 4-bit pages, drawn on the CPU, garbage wherever no row is."""
import numpy as np
import torch

import page_reference as ref
import paper_2605_30574_amd as sp
from gpu_common import announce

P = 64
BF16 = 2.0 ** -8          # half a step of bfloat16
FILL = 776.0              # exact in bfloat16


# (donor, window): (D, (Hq, Hkv), T, C, T_p) whose prompts are walked by tiles of several cells' rows
SHARED = {
    ("diff", 0): [(64, (16, 8), 1, 16, 3000), (64, (16, 4), 5, 16, 3000), (128, (16, 8), 1, 16, 3000), (128, (16, 4), 5, 16, 3000),
                  (256, (16, 8), 1, 16, 3000), (128, (8, 2), 1, 160, 3000)],
    ("diff", 2000): [(64, (16, 8), 1, 80, 1500), (64, (8, 2), 5, 160, 1500), (128, (16, 8), 1, 16, 3000), (128, (8, 2), 5, 120, 1500),
                     (256, (16, 8), 1, 16, 3000)],
    ("zero", 0): [(64, (16, 8), 2, 16, 5000), (64, (16, 4), 5, 16, 5000), (128, (16, 8), 1, 16, 5000), (128, (16, 4), 5, 16, 5000),
                  (256, (16, 8), 1, 40, 1500)],
    ("zero", 2000): [(64, (16, 8), 1, 120, 1500), (128, (16, 8), 1, 16, 5000), (128, (8, 2), 5, 80, 3000), (256, (16, 8), 1, 40, 1500)],
}


def shared_case(D, heads, T, C, Tp):
    """Arguments of Sweep: cells at two steps, not spliced, spliced, or from the middle of their tokens on."""
    steps = [60 if c % 2 else 5 for c in range(C)]
    return dict(C=C, T=T, Hq=heads[0], Hkv=heads[1], D=D, Tp=Tp, span=(70, Tp // 2), cap=80, steps=steps,
                LW=[([9, 0], [0, 0], [1, steps[c] + T // 2])[c % 3] for c in range(C)])


# ... with finished cells, cells without tokens and others with fewer than T among them: (donor, window, D, (Hq, Hkv), T, C, T_p)
RAGGED = [("diff", 0, 64, (16, 8), 2, 60, 3000), ("diff", 0, 128, (16, 8), 1, 40, 3000), ("zero", 0, 128, (16, 4), 6, 40, 5000),
          ("diff", 2000, 128, (8, 2), 5, 120, 3000), ("diff", 0, 256, (16, 8), 2, 40, 3000), ("zero", 2000, 256, (16, 8), 2, 80, 3000)]


def ragged_case(donor, window, D, heads, T, C, Tp):
    """Arguments of Sweep: every cell at a step of its own, every fifth finished, 0 to T tokens."""
    steps = np.array([-1 if c % 5 == 3 else 7 * c % 73 for c in range(C)])
    return dict(donor=donor, window=window, C=C, T=T, Hq=heads[0], Hkv=heads[1], D=D, Tp=Tp, span=(70, Tp // 2), cap=80, steps=steps,
                new=np.array([T - c % 4 * T // 3 if c % 7 else 0 for c in range(C)]),
                LW=[([9, 0], [0, 0], [1, max(int(steps[c]), 0) + T // 2])[c % 3] for c in range(C)])


class Sweep:
    """One call's tensors on the GPU and their float64 values."""

    def __init__(self, seed, C=3, T=1, Hq=8, Hkv=2, D=64, Tp=37, span=(5, 30), cap=100, donor="diff", window=0, layer=1, n_layers=4,
                 steps=None, new=None, LW=None, scale=None, spread=1.0, extra=2):
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.C, self.T, self.Hq, self.Hkv, self.D, self.Tp, self.span, self.cap = C, T, Hq, Hkv, D, Tp, span, cap
        self.window, self.layer, self.zero = window, layer, donor == "zero"
        self.scale = D ** -0.5 if scale is None else scale
        self.steps = np.asarray(rng.integers(0, cap - T + 1, C) if steps is None else steps, np.int32)
        self.new = None if new is None else np.asarray(new, np.int32)
        self.LW = np.asarray([[int(rng.integers(0, n_layers + 1)), int(rng.integers(0, cap))] for _ in range(C)]
                             if LW is None else LW, np.int32)
        L, Lp = -(-cap // P), -(-Tp // P)
        self.L = L
        order = rng.permutation(C * L + 2 * Lp + extra)
        self.n_pages = len(order)
        self.tables = order[:C * L].reshape(C, L).astype(np.int32)
        self.clean, self.donor = order[C * L:C * L + Lp].astype(np.int32), order[C * L + Lp:C * L + 2 * Lp].astype(np.int32)
        self.pool = rng.integers(0, 256, (self.n_pages, Hkv, ref.head_bytes(D)), dtype=np.uint8)
        self.rows = {}            # page -> (k, v) [Hkv][64][D]
        count = self.counts()
        for c in range(C):
            for j in range(L):
                # rows behind the cell's last one are garbage, NaN bytes among them
                self.fill(self.tables[c, j], max(0, min(P, int(self.steps[c]) + int(count[c]) - j * P)), spread)
        for j in range(Lp):
            for page in (self.clean[j], self.donor[j]):
                self.fill(page, min(P, Tp - j * P), spread, sink=j == 0)
        self.q = torch.from_numpy(rng.standard_normal((C, T, Hq, D))).to(torch.bfloat16)
        self.shape = sp.make_shape(C, n_layers, Hq, Hkv, D, Tp, span, cap, self.zero, "bf16")
        self.pages = sp.make_pages(self.n_pages, L, T)
        self.call = sp.make_call(layer, 0, window, self.scale)

    def counts(self):
        n = np.full(self.C, self.T) if self.new is None else self.new
        return np.where(self.steps >= 0, n, 0)

    def fill(self, page, n, spread=1.0, sink=False):
        """n rows of a page drawn, the others left as garbage."""
        D = self.D
        for h in range(self.Hkv):
            if n <= 0:
                continue
            k, v = (self.rng.standard_normal((P, D)) * 2.0 ** self.rng.uniform(-spread, spread, (P, 1)) for _ in range(2))
            if sink:
                k[0, :4] *= 50
            self.put(page, h, k, v, range(n))

    def put(self, page, h, k, v, rows):
        """Rows of k, v [64][D] stored in a page."""
        at, new = ref.places(np.arange(P)[:, None], np.arange(self.D), self.D), ref.page_of(k, v)
        rows = np.asarray(list(rows))
        for x in at:
            i = np.broadcast_to(x, (P, self.D))[rows]
            self.pool[page, h][i] = new[i]

    def stored(self, table, n, h):
        """(k, v) of rows 0..n-1 under a table; rows of absent pages are None."""
        k, v = np.full((n, self.D), np.nan), np.full((n, self.D), np.nan)
        there = np.zeros(n, bool)
        for j in range(-(-n // P)):
            page, m = int(table[j]), min(P, n - j * P)
            if 0 <= page < self.n_pages:
                a, b = ref.rows_of(self.pool[page, h], self.D)
                k[j * P:j * P + m], v[j * P:j * P + m], there[j * P:j * P + m] = a[:m], b[:m], True
        return k, v, there

    def send(self):
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.dev = dict(tables=up(self.tables), clean=up(self.clean), donor=None if self.zero else up(self.donor),
                        pool=up(self.pool.reshape(self.n_pages, -1)), q=self.q.cuda())

    def attend(self, split=0, ws=None, stream=None, send=True):
        if send:
            self.send()
        d = self.dev
        self.call.split_keys = split
        out = torch.full((self.C, self.T, self.Hq, self.D), FILL, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.C, self.T, self.Hq), FILL, device="cuda")
        if ws is None:
            ws = torch.empty(sp.splice_page_attn_workspace_bytes(self.shape, self.call, self.pages), dtype=torch.uint8, device="cuda")
        sp.splice_page_attn(self.shape, self.call, self.pages, self.LW, self.steps, self.new, d["tables"], d["clean"], d["donor"],
                            d["q"], d["pool"], out, lse, ws, stream)
        torch.cuda.synchronize()
        return out, lse

    def expected(self):
        """(out, lse, out's tolerance, lse's) float64.

        A score is a sum of D exact products in fp32: off by D + 4 steps of sum |q||k| at most, times the scale.  The weights
        are off by that, by 4 steps in exp2 and its argument's (relative to the largest score and to itself) and, as
        bf16, by 2^-8; the values' sum and the weights' by a step a key.  The result is rounded once more."""
        C, T, Hq, Hkv, D, Tp = self.C, self.T, self.Hq, self.Hkv, self.D, self.Tp
        G, count = Hq // Hkv, self.counts()
        q = self.q.double().numpy()
        out, lse = np.full((C, T, Hq, D), FILL), np.full((C, T, Hq), FILL)
        tol_o, tol_l = np.zeros((C, T, Hq, D)), np.zeros((C, T, Hq))
        eps = 2.0 ** -23
        prompts = {}
        for h in range(Hkv):
            prompts[h] = [self.stored(self.clean, Tp, h), None if self.zero else self.stored(self.donor, Tp, h)]
        a, b = self.span
        for c in range(C):
            for h in range(Hkv):
                if count[c] == 0:
                    continue
                s0 = int(self.steps[c])
                gk, gv, gt = self.stored(self.tables[c], s0 + int(count[c]), h)
                for t in range(int(count[c])):
                    step, pos = s0 + t, Tp + s0 + t
                    (k, v, there), donor = prompts[h]
                    k, v, there = k.copy(), v.copy(), there.copy()
                    if self.layer >= self.LW[c, 0] and step >= self.LW[c, 1]:
                        if self.zero:
                            k[a:b], v[a:b], there[a:b] = 0, 0, True
                        else:
                            for x, y in zip((k, v, there), donor):
                                x[a:b] = y[a:b]
                    low = max(0, pos - self.window + 1) if self.window else 0
                    k, v, there = (np.concatenate([x, y])[low:pos + 1] for x, y in ((k, gk), (v, gv), (there, gt)))
                    k, v = k[there], v[there]
                    for g in range(G):
                        i = (c, t, h * G + g)
                        o, z, weight, score = ref.attend(q[i], k, v, self.scale)
                        out[i], lse[i] = o, z
                        err = (D + 4) * eps * score + 4 * eps * (1 + 2 * score)
                        tol_o[i] = BF16 * (weight + np.abs(o)) * 1.01 + (2 * err + 2 * (len(k) + 8) * eps) * weight + 2.0 ** -126
                        tol_l[i] = err + (len(k) + 8) * eps + 4 * eps * (abs(z) if np.isfinite(z) else 0)
        return out, lse, tol_o, tol_l

    def check(self, out, lse, what=""):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        wo, wl, to, tl = self.expected()
        for name, x, y, t in (("out", out, wo, to), ("lse", lse, wl, tl)):
            same = (x == y) | (np.isnan(x) & np.isnan(y))
            with np.errstate(invalid="ignore"):
                bad = ~(same | (np.abs(x - y) <= t))
            assert not bad.any(), f"{what} {name}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: " \
                                  f"{x[bad][0]} for {y[bad][0]}, tolerance {t[bad][0]}"
