"""Inputs of the tree operators' GPU tests: small sweeps with random trees, drawn on the CPU."""
import numpy as np
import torch

import paper_2605_30574_amd as sp
from gpu_common import announce
import tree_reference as ref

F64 = torch.float64


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def random_parents(rng, C, T, padded=True):
    p = np.full((C, T), -2, np.int64)
    for c in range(C):
        n = T if not padded or c % 2 else int(rng.integers(1, T + 1))
        for t in range(n):
            p[c, t] = -1 if t == 0 or rng.random() < 0.1 else int(rng.integers(max(0, t - 3), t))
    return p


class Sweep:
    """One call's tensors on the GPU and their float64 values."""

    def __init__(self, seed, C=3, T=5, Hq=8, Hkv=2, D=64, Tp=37, span=(5, 30), cap=40, kv="bf16", donor="diff", window=0,
                 layer=1, n_layers=4, steps=None, LW=None, scale=None, parents=None):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.C, self.T, self.Hq, self.Hkv, self.D, self.Tp, self.span, self.cap = C, T, Hq, Hkv, D, Tp, span, cap
        self.kv, self.window, self.layer = kv, window, layer
        self.scale = D ** -0.5 if scale is None else scale
        self.steps = np.asarray(rng.integers(0, cap - T + 1, C) if steps is None else steps, np.int32)
        self.LW = np.asarray([[int(rng.integers(0, n_layers + 1)), int(rng.integers(0, cap))] for _ in range(C)]
                             if LW is None else LW, np.int32)
        self.depth, self.visible = sp.tree_layout(random_parents(rng, C, T) if parents is None else parents)
        bf = torch.bfloat16
        self.q = randn(C, T, Hq, D).to(bf).cuda()
        self.clean = [randn(Hkv, Tp, D) for _ in range(2)]
        if Tp:
            self.clean[0][:, 0, :4] *= 50
        self.clean = [x.to(bf).cuda() for x in self.clean]
        self.donor = [None, None] if donor == "zero" else [randn(Hkv, Tp, D).to(bf).cuda() for _ in range(2)]
        x = [randn(C, Hkv, cap, D) for _ in range(2)]
        if kv == "bf16":
            self.gen, self.exps = [y.to(bf).cuda() for y in x], [None, None]
        else:
            codes = [ref.quantised(y.double().numpy()) for y in x]
            self.gen = [torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda() for v, _ in codes]
            self.exps = [torch.from_numpy((e + 127).astype(np.uint8)).cuda() for _, e in codes]
        self.shape = sp.make_shape(C, n_layers, Hq, Hkv, D, Tp, span, cap, donor == "zero", "bf16")
        self.tree = sp.make_tree(T, kv)
        self.send_tree()

    def send_tree(self):
        self.depth_dev = torch.from_numpy(self.depth).cuda()
        self.visible_dev = torch.from_numpy(self.visible.view(np.int64)).cuda()

    def gen_values(self):
        if self.kv == "bf16":
            return [f64(x) for x in self.gen]
        return [f64(x.view(torch.float8_e4m3fn).float()) * np.exp2(f64(e) - 127)[..., None] for x, e in zip(self.gen, self.exps)]

    def call(self, split=0):
        return sp.make_call(self.layer, 0, self.window, self.scale, split)

    def outputs(self):
        return (torch.full((self.C, self.T, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((self.C, self.T, self.Hq), 7.0, device="cuda"))

    def workspace(self, split=0):
        n = sp.splice_tree_attn_workspace_bytes(self.shape, self.call(split), self.tree)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # NaN wherever nothing is written

    def attend(self, split=0, out=None, lse=None, workspace=None, stream=None):
        if out is None:
            out, lse = self.outputs()
        ws = self.workspace(split) if workspace is None else workspace
        sp.splice_tree_attn(self.shape, self.call(split), self.tree, self.LW, self.steps, self.depth_dev, self.visible_dev,
                            self.q, *self.clean, *self.donor, *self.gen, *self.exps, out, lse, ws, stream)
        return out, lse

    def expected(self):
        donor = None if self.donor[0] is None else [f64(x) for x in self.donor]
        return ref.attention(f64(self.q), [f64(x) for x in self.clean], donor, self.gen_values(), self.depth, self.visible,
                             self.steps, self.LW, self.layer, self.window, self.scale, self.span)

    def check(self, out, lse, what=""):
        torch.cuda.synchronize()
        want, want_lse, spread, size, n = self.expected()
        computed = ~np.isnan(want_lse)
        tol, tol_lse = ref.attention_bounds(want, want_lse, spread, size, n, self.D)
        o, l = f64(out), f64(lse)
        assert (o[~computed] == 7.0).all() and (l[~computed] == 7.0).all(), f"{what}: rows that are not the call's were written"
        assert np.isfinite(o[computed]).all(), f"{what}: not finite"
        off = np.abs(o - want)[computed] - tol[computed]
        assert (off <= 0).all(), f"{what}: out off by {off.max():.3e} more than it may be, at {np.argwhere(off > 0)[:4].tolist()}"
        empty = np.isneginf(want_lse)
        assert (l[empty] == -np.inf).all() and (o[empty] == 0).all(), f"{what}: a row that sees nothing"
        full = computed & ~empty
        assert (np.abs(l - want_lse)[full] <= tol_lse[full]).all(), f"{what}: lse"


__all__ = ["Sweep", "announce", "f64", "random_parents", "ref", "sp"]
