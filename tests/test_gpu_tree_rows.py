"""splice_tree_append, splice_tree_read and splice_tree_keep against the definitions in float64."""
import numpy as np
import pytest
import torch

from tree_common import announce, f64, random_parents, ref, sp

pytestmark = pytest.mark.gpu


class Rows:
    def __init__(self, seed, C=4, T=6, Hq=8, Hkv=2, D=64, Tp=100, cap=30, kv="bf16", steps=None, fused=True, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.C, self.T, self.Hq, self.Hkv, self.D, self.Tp, self.cap, self.kv = C, T, Hq, Hkv, D, Tp, cap, kv
        self.steps = np.asarray([0, cap - T, -1, 5][:C] if steps is None else steps, np.int32)
        self.depth, _ = sp.tree_layout(random_parents(rng, C, T))
        self.depth_dev = torch.from_numpy(self.depth).cuda()
        if fused:
            qkv = (torch.randn(C, T, (Hq + 2 * Hkv) * D, generator=g) * spread).to(torch.bfloat16).cuda()
            self.q, self.k, self.v = (x.unflatten(2, (-1, D)) for x in qkv.split((Hq * D, Hkv * D, Hkv * D), dim=2))
        else:
            self.q, self.k, self.v = ((torch.randn(C, T, n, D, generator=g) * spread).to(torch.bfloat16).cuda()
                                      for n in (Hq, Hkv, Hkv))
        shape = (C, Hkv, cap, D)
        if kv == "bf16":
            self.gen = [torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
            self.exps = [None, None]
        else:
            self.gen = [torch.randint(0, 127, shape, generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
            self.exps = [torch.randint(100, 140, shape[:3], generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
        self.q_out = torch.full((C, T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.shape = sp.make_shape(C, 1, Hq, Hkv, D, Tp, (0, 0), cap, True, "bf16")
        self.tree = sp.make_tree(T, kv)

    def written(self):
        return (self.depth >= 0) & (self.steps[:, None] >= 0)

    def values(self):
        if self.kv == "bf16":
            return [f64(x) for x in self.gen]
        return [f64(x.view(torch.float8_e4m3fn).float()) * np.exp2(f64(e) - 127)[..., None] for x, e in zip(self.gen, self.exps)]

    def append(self, rope, freq, **kw):
        sp.splice_tree_append(self.shape, self.tree, rope, freq, self.steps, self.depth_dev, self.q, self.k, self.v, self.q_out,
                              *self.gen, *self.exps, **kw)
        torch.cuda.synchronize()


def near(got, want, tol):
    off = np.abs(got - want) - tol
    assert (off <= 0).all(), f"off by {off.max():.3e} more than it may be"


# the rotation in fp32: cos and sin to 2 ulp of 1 (2^-22 each), two products and a sum (3 * 2^-24), of values |a| + |b|
ROT = 2.0 ** -21


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,R", [((8, 2, 64), 64), ((8, 2, 64), 16), ((8, 2, 64), 0), ((4, 4, 128), 128), ((16, 2, 128), 96),
                                     ((3, 3, 256), 256), ((8, 1, 256), 64)])
def test_append(heads, R, layout, kv):
    Hq, Hkv, D = heads
    if Hq == 3:
        Hq, Hkv = 4, 4
    mscale = 1.0 if layout == "half" else 1.25
    r = Rows(R + D, Hq=Hq, Hkv=Hkv, D=D, kv=kv, fused=layout == "half", Tp=100000)
    announce(f"append {heads} R={R} {layout} {kv}")
    freq = 10000.0 ** (-np.arange(0, R, 2) / max(R, 1))
    before, exps = [x.clone() for x in r.gen], [None if e is None else e.clone() for e in r.exps]
    r.append(sp.make_rope(layout, R, mscale), torch.from_numpy(freq).cuda() if R else None)
    on = r.written()
    pos = r.Tp + r.steps[:, None].astype(np.int64) + r.depth
    turned = {}
    for name, x in (("q", r.q), ("k", r.k)):
        y = f64(x)
        heads_pos = np.broadcast_to(pos[..., None], y.shape[:3])
        turned[name] = (ref.rotated(y, heads_pos, freq, layout, R, mscale), ref.rotated(np.abs(y), heads_pos * 0, freq, layout, R, mscale))
        turned[name] += (np.abs(y).max(-1, keepdims=True) * 2 * mscale,)
    q = f64(r.q_out)
    assert (q[~on] == 7.0).all()
    want, _, size = turned["q"]
    near(q[on], want[on], (2.0 ** -8 * np.abs(want) + ROT * size + 2.0 ** -126)[on])
    got = r.values()
    for n, (want, size) in enumerate(((turned["k"][0], turned["k"][2]), (f64(r.v), None))):
        touched = np.zeros((r.C, r.cap), bool)
        for c, t in np.argwhere(on):
            row = r.steps[c] + t
            touched[c, row] = True
            w = want[c, t]
            if kv == "bf16":
                tol = 2.0 ** -8 * np.abs(w) + (0 if size is None else ROT * size[c, t]) + 2.0 ** -126 if n == 0 else 0.0 * w
                near(got[n][c, :, row], w, tol)
            elif n == 1:   # not rotated: the very codes and exponents
                code, e = ref.quantised(w)
                assert np.array_equal(got[n][c, :, row], np.ldexp(code, e[..., None]))
                assert np.array_equal(f64(r.exps[n])[c, :, row], e + 127)
            else:          # half a step of the larger exponent that the rotation's error may reach
                top = (np.abs(w).max(-1, keepdims=True) + ROT * size[c, t])
                _, e = ref.quantised(np.repeat(top, 2, -1))
                near(got[n][c, :, row], w, 2.0 ** -4 * np.abs(w) + np.exp2(e - 10.0)[..., None] + ROT * size[c, t] * (1 + 2.0 ** -4))
        keep = torch.from_numpy(~touched).cuda()
        assert torch.equal(r.gen[n].transpose(1, 2)[keep], before[n].transpose(1, 2)[keep])
        if kv == "e4m3":
            assert torch.equal(r.exps[n].transpose(1, 2)[keep], exps[n].transpose(1, 2)[keep])


def test_append_given_positions_in_place():
    r = Rows(5, fused=False, T=3)
    pos = torch.randint(0, 1 << 31, (r.C, r.T), generator=torch.Generator().manual_seed(1)).cuda()
    freq = 5e5 ** (-np.arange(0, 64, 2) / 64)
    y = f64(r.q)
    r.q_out = r.q
    r.append(sp.make_rope("half", 64), torch.from_numpy(freq).cuda(), pos=pos)
    want = ref.rotated(y, np.broadcast_to(f64(pos)[..., None], y.shape[:3]), freq, "half", 64, 1.0)
    on = r.written()
    want[~on] = y[~on]
    # 2^31 * freq in 64 bits: an angle is off by 2^31 * 2^-52
    near(f64(r.q), want, 2.0 ** -8 * np.abs(want) + (ROT + 2.0 ** -20) * np.abs(y).max(-1, keepdims=True) * 2)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_quantised_rows_of_every_size(D):
    """Rows from 2^-133 to 2^127, with zeros, values at the borders between two codes, and non-finite ones."""
    C, T, Hkv = 2, 64, 2
    r = Rows(9, C=C, T=T, Hq=2, Hkv=Hkv, D=D, cap=70, kv="e4m3", steps=[0, 6], fused=False)
    r.depth[:] = 0
    r.depth_dev = torch.from_numpy(r.depth).cuda()
    x = f64(r.v)
    for t in range(T):
        x[0, t] *= 2.0 ** (-133 + 4 * t)
    x[1, :8, :, :] = np.clip(np.rint(x[1, :8] * 16) / 16, -1.75, 1.75)
    x[1, 8] = 0.0
    x[1, 9, 0] = 448.0
    x[1, 10, :, :4] = 2.0 ** -9 * np.array([0.5, 1.5, 2.5, 1.0])
    x[1, 10, :, 4] = 448.0
    x[1, 11, 0, 3] = np.inf
    x[1, 12, 1, 5] = np.nan
    x[1, 13, 0, D - 1] = -np.inf
    x[1, 14, 0] = 3.38953139e38   # the largest bf16 number
    r.v = torch.from_numpy(x).to(torch.bfloat16).cuda()
    x = f64(r.v)
    r.append(sp.make_rope("half", 0), None)
    rows = [torch.empty(C, Hkv, T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sp.splice_tree_read(r.shape, r.tree, r.steps, *r.gen, *r.exps, *rows)
    torch.cuda.synchronize()
    got = f64(rows[1]).transpose(0, 2, 1, 3)
    with np.errstate(all="ignore"):
        code, e = ref.quantised(x)
        want = np.ldexp(np.clip(code, -np.where(e >= 120, 240, 448)[..., None], np.where(e >= 120, 240, 448)[..., None]), e[..., None])
    bad = ~np.isfinite(x).all(-1)
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad])
    assert np.isfinite(got[~bad]).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,D", [(1, 64), (7, 128), (64, 64), (64, 128), (64, 256)])
def test_read_and_keep(T, D, kv):
    C = 5
    r = Rows(T + D, C=C, T=T, D=D, cap=T + 9, kv=kv, steps=[0, 9, -1, 4, 2])
    rng = np.random.default_rng(T)
    rows = [torch.full((C, r.Hkv, T, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    announce(f"read {T} {D} {kv}")
    sp.splice_tree_read(r.shape, r.tree, r.steps, *r.gen, *r.exps, *rows)
    torch.cuda.synchronize()
    before = r.values()
    for n in range(2):
        for c in range(C):
            s = int(r.steps[c])
            want = np.full((r.Hkv, T, D), 7.0) if s < 0 else before[n][c, :, s:s + T]
            assert np.array_equal(f64(rows[n])[c], want)
    keep = np.full((C, T), -1, np.int32)
    count = np.zeros(C, int)
    for c in range(C):
        count[c] = int(rng.integers(0, T + 1))
        keep[c, :count[c]] = np.sort(rng.choice(T, size=count[c], replace=False))
    keep[1] = np.arange(T)                       # all of them: nothing moves
    count[1] = T
    if T >= 7:
        keep[3] = -1
        keep[3, :5] = [1, 3, 3, 4, 5]            # ends at the entry that does not ascend
        keep[4] = -1
        keep[4, :4] = [2, 5, T, 6]               # ends at the entry that is no node
        count[3], count[4] = 2, 2
    announce(f"keep {T} {D} {kv}")
    sp.splice_tree_keep(r.shape, r.tree, r.steps, torch.from_numpy(keep).cuda(), *r.gen, *r.exps)
    torch.cuda.synchronize()
    after = r.values()
    for n in range(2):
        want = before[n].copy()
        for c in range(C):
            s = int(r.steps[c])
            if s >= 0:
                want[c, :, s:s + count[c]] = \
                    before[n][c][:, s + keep[c, :count[c]]]
        assert np.array_equal(after[n], want)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_captured_append_attend_keep(kv):
    """A pass's calls in one graph, replayed on new inputs between eager work: the bits of eager calls."""
    s = Rows(31, C=4, T=6, D=64, Tp=100, cap=40, kv=kv, fused=False)
    g = torch.Generator().manual_seed(32)
    bf = torch.bfloat16
    randn = lambda *shape: torch.randn(*shape, generator=g).to(bf).cuda()  # noqa: E731
    shape = sp.make_shape(s.C, 4, s.Hq, s.Hkv, s.D, s.Tp, (10, 70), s.cap, False, "bf16")
    prompt = [randn(s.Hkv, s.Tp, s.D) for _ in range(4)]
    call, rope = sp.make_call(1, 0, 0, s.D ** -0.5, 64), sp.make_rope("half", s.D)
    freq = torch.from_numpy(sp.rope_frequencies(s.D, 1e4)[0]).cuda()
    _, visible = sp.tree_layout(random_parents(np.random.default_rng(31), s.C, s.T))
    visible = torch.from_numpy(visible.view(np.int64)).cuda()
    keep = torch.tensor([[0, 2, 5, -1, -1, -1], [1, 3, -1, -1, -1, -1], [-1] * 6, [0, 1, 2, 3, 4, 5]], dtype=torch.int32).cuda()
    lw = np.array([[0, 0], [0, 8], [9, 0], [1, 6]], np.int32)
    start = [x.clone() for x in s.gen]
    start_e = [None if x is None else x.clone() for x in s.exps]

    def buffers():
        n = sp.splice_tree_attn_workspace_bytes(shape, call, s.tree)
        return dict(q=torch.zeros_like(s.q_out), gen=[x.clone() for x in start], e=[None if x is None else x.clone() for x in start_e],
                    out=torch.zeros_like(s.q_out), lse=torch.zeros(s.C, s.T, s.Hq, device="cuda"),
                    ws=torch.empty(n, dtype=torch.uint8, device="cuda"))

    def calls(b):
        sp.splice_tree_append(shape, s.tree, rope, freq, s.steps, s.depth_dev, s.q, s.k, s.v, b["q"], *b["gen"], *b["e"])
        sp.splice_tree_attn(shape, call, s.tree, lw, s.steps, s.depth_dev, visible, b["q"], *prompt, *b["gen"], *b["e"], b["out"],
                            b["lse"], b["ws"])
        sp.splice_tree_keep(shape, s.tree, s.steps, keep, *b["gen"], *b["e"])

    cap = buffers()
    calls(cap)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(cap)
    for n in range(4):
        announce(f"captured pass {kv}, replay {n}")
        for x in (s.q, s.k, s.v):
            x.copy_(randn(*x.shape))
        for x, y in zip(cap["gen"] + cap["e"], start + start_e):
            if x is not None:
                x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        eager = buffers()
        calls(eager)
        torch.cuda.synchronize()
        for name in ("q", "out", "lse"):
            assert torch.equal(cap[name], eager[name]), name
        for x, y in zip(cap["gen"] + cap["e"], eager["gen"] + eager["e"]):
            assert x is None or torch.equal(x, y)


@pytest.mark.parametrize("layout,D,R", [("half", 128, 128), ("interleaved", 128, 64), ("half", 64, 64), ("interleaved", 256, 256)])
def test_codes_are_those_of_the_rotation_in_64_bits(layout, D, R):
    """A million rotated values: every code and exponent, those next to a border too (a rotation in fp32 has some of them wrong).
    The kernel's angles and its series are off by some 2^-33, which no border here is as near as."""
    r = Rows(41 + D, C=4, T=64, Hq=16 * 128 // D, Hkv=16 * 128 // D, D=D, cap=80, Tp=50000, kv="e4m3", steps=[0, 16, 3, 7], fused=False)
    freq = 1e6 ** (-np.arange(0, R, 2) / R) / 8
    r.append(sp.make_rope(layout, R, 1.1), torch.from_numpy(freq).cuda())
    y = f64(r.k)
    pos = np.broadcast_to((r.Tp + r.steps[:, None].astype(np.int64) + r.depth)[..., None], y.shape[:3])
    code, e = ref.quantised(ref.rotated(y, pos, freq, layout, R, 1.1))
    got, exps, on = r.values()[0], f64(r.exps[0]), r.written()
    wrong = 0
    for c, t in np.argwhere(on):
        row = r.steps[c] + t
        assert np.array_equal(exps[c, :, row], e[c, t] + 127)
        wrong += int((got[c, :, row] != np.ldexp(code[c, t], e[c, t][..., None])).sum())
    assert wrong == 0


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("C,finished", [(32, 0), (33, 0), (40, 8), (41, 8), (256, 0), (256, 100)])
def test_many_cells(C, finished, kv):
    """Rows of up to as many cells as a call takes, some finished: appended unturned, read back, the second node kept as the first."""
    rng = np.random.default_rng(C + finished)
    steps = rng.integers(0, 9, C).astype(np.int32)
    steps[rng.choice(C, finished, replace=False)] = -1
    r = Rows(51, C=C, T=3, cap=11, kv=kv, steps=steps, fused=False)
    r.depth[:] = np.arange(3)
    r.depth_dev = torch.from_numpy(r.depth).cuda()
    start = [x.clone() for x in r.gen]
    r.append(sp.make_rope("half", 0), None)
    rows = [torch.full((C, r.Hkv, 3, r.D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sp.splice_tree_read(r.shape, r.tree, r.steps, *r.gen, *r.exps, *rows)
    torch.cuda.synchronize()
    on = torch.from_numpy(steps >= 0).cuda()
    for got, x, cache, before in zip(rows, (r.k, r.v), r.gen, start):
        want = x.transpose(1, 2)
        if kv == "bf16":
            assert torch.equal(got[on], want[on])
        else:
            code, e = ref.quantised(f64(want))
            assert np.array_equal(f64(got)[steps >= 0], np.ldexp(code, e[..., None])[steps >= 0])
        assert (got[~on] == 5.0).all() and torch.equal(cache[~on], before[~on])
    kept = [x.clone() for x in r.gen]
    keep = torch.tensor([[1, 2, -1]] * C, dtype=torch.int32).cuda()
    sp.splice_tree_keep(r.shape, r.tree, r.steps, keep, *r.gen, *r.exps)
    torch.cuda.synchronize()
    for x, y in zip(r.gen, kept):
        for c in range(C):
            s = steps[c]
            if s >= 0:
                y[c, :, s:s + 2] = y[c, :, s + 1:s + 3].clone()
        assert torch.equal(x, y)
