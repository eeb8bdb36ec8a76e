"""splice_page_append and splice_page_read against the definitions in float64."""
import numpy as np
import pytest
import torch

import page_reference as ref
import paper_2605_30574_amd as sp
from gpu_common import announce

pytestmark = pytest.mark.gpu
P, FILL = 64, 776.0   # (exact in bfloat16)


def turned(x, pos, freq, layout, mscale):
    """Rotary positions in float64: x [..., D], pos [...], freq [R / 2]."""
    R = 2 * len(freq)
    ang = pos[..., None] * freq
    c, s = np.cos(ang) * mscale, np.sin(ang) * mscale
    y = x.copy()
    if layout == "half":
        u, w = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = u * c - w * s, w * c + u * s
    else:
        u, w = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = u * c - w * s, w * c + u * s
    return y


class Rows:
    def __init__(self, seed, C=3, T=4, Hq=8, Hkv=2, D=64, cap=200, Tp=33, steps=None, new=None, spread=3.0, extra=3):
        rng = np.random.default_rng(seed)
        self.C, self.T, self.Hq, self.Hkv, self.D, self.Tp = C, T, Hq, Hkv, D, Tp
        L = -(-cap // P)
        self.n_pages = C * L + extra
        self.tables = rng.permutation(self.n_pages)[:C * L].reshape(C, L).astype(np.int32)
        self.steps = np.asarray(rng.integers(0, cap - T + 1, C) if steps is None else steps, np.int32)
        self.new = None if new is None else np.asarray(new, np.int32)
        self.count = np.where(self.steps >= 0, T if new is None else self.new, 0)
        self.pool = rng.integers(0, 256, (self.n_pages, Hkv, ref.head_bytes(D)), dtype=np.uint8)
        draw = lambda h: torch.from_numpy(rng.standard_normal((C, T, h, D)) * 2.0 ** rng.uniform(-spread, spread, (C, T, h, D))).to(torch.bfloat16)  # noqa: E731
        self.q, self.k, self.v = draw(Hq), draw(Hkv), draw(Hkv)
        self.shape = sp.make_shape(C, 1, Hq, Hkv, D, Tp, (0, 0), cap, False, "bf16")
        self.pages = sp.make_pages(self.n_pages, L, T)

    def run(self, layout="half", rotary=None, theta=1e4, mscale=1.0, pos=None, fused=False, stream=None):
        R = self.D if rotary is None else rotary
        self.freq = theta ** (-np.arange(0, R, 2) / max(R, 1))
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.tab, self.mem = up(self.tables), up(self.pool.reshape(self.n_pages, -1))
        q, k, v = self.q.cuda(), self.k.cuda(), self.v.cuda()
        if fused:   # parts of one projection's rows
            both = torch.cat([x.flatten(2) for x in (q, k, v)], -1)
            q, k, v = (x.unflatten(2, (-1, self.D)) for x in both.split([x.shape[2] * self.D for x in (q, k, v)], -1))
        out = torch.full((self.C, self.T, self.Hq, self.D), FILL, dtype=torch.bfloat16, device="cuda")
        sp.splice_page_append(self.shape, self.pages, sp.make_rope(layout, R, mscale), up(self.freq) if R else None, self.steps, self.new,
                              self.tab, q, k, v, out, self.mem, None if pos is None else up(pos), stream)
        torch.cuda.synchronize()
        at = self.Tp + self.steps[:, None] + np.arange(self.T) if pos is None else pos
        at = np.broadcast_to(at, (self.C, self.T))[:, :, None].astype(float)
        turn = lambda x: turned(x.double().numpy(), at, self.freq, layout, mscale)  # noqa: E731
        return out, turn(self.q), turn(self.k), self.v.double().numpy()

    def check(self, out, q, k, v, what=""):
        """q to half a step of bfloat16 (and fp32's roundings of a rotation), the codes and every other byte exactly."""
        want, got = np.full(q.shape, FILL), out.double().cpu().numpy()
        pool = self.pool.copy()
        for c in range(self.C):
            n = int(self.count[c])
            want[c, :n] = q[c, :n]
            for t in range(n):
                r = int(self.steps[c]) + t
                page = self.tables[c, r // P]
                if not 0 <= page < self.n_pages:
                    continue
                kb, vb, ks, vs = ref.places(r % P, np.arange(self.D), self.D)
                for h in range(self.Hkv):
                    bad = not (np.isfinite(k[c, t, h]).all() and np.isfinite(v[c, t, h]).all())
                    for x, code_at, scale_at in ((k[c, t, h], kb, ks), (v[c, t, h], vb, vs)):
                        codes, e = (np.zeros(self.D, int), np.full(self.D // 32, 128)) if bad else ref.quantised(x)
                        pool[page, h, code_at[0::2]] = codes[0::2] + 16 * codes[1::2]
                        pool[page, h, scale_at[0::32]] = e + 127
        size = np.sqrt((np.where(np.isfinite(q), q, 0) ** 2).sum(-1, keepdims=True))
        ok = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * size)
        assert ok.all(), f"{what}: q off at {np.argwhere(~ok)[0]}"
        mem = self.mem.cpu().numpy().reshape(pool.shape)
        assert (mem == pool).all(), f"{what}: {(mem != pool).sum()} bytes off, first at {np.argwhere(mem != pool)[0]}"
        return pool

    def read(self):
        shape = (self.C, self.Hkv, self.T, self.D)
        rows = [torch.full(shape, FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        sp.splice_page_read(self.shape, self.pages, self.steps, self.new, self.tab, self.mem, *rows)
        torch.cuda.synchronize()
        return [x.double().cpu().numpy() for x in rows]

    def check_read(self, pool, what=""):
        got = self.read()
        want = [np.full(got[0].shape, FILL) for _ in range(2)]
        for c in range(self.C):
            for t in range(int(self.count[c])):
                r = int(self.steps[c]) + t
                page = self.tables[c, r // P]
                if 0 <= page < self.n_pages:
                    for h in range(self.Hkv):
                        kv = ref.rows_of(pool[page, h], self.D)
                        for w, x in zip(want, kv):
                            w[c, h, t] = x[r % P]
        for g, w, name in zip(got, want, "kv"):
            ok = (g == w) | (np.isnan(g) & np.isnan(w))
            assert ok.all(), f"{what} rows of {name}: first at {np.argwhere(~ok)[0]}"


HEADS = [(8, 2, 64), (3, 3, 64), (8, 1, 128), (32, 8, 128), (2, 2, 256), (8, 4, 256)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("T", [1, 5, 70])
def test_heads_layouts_and_tokens(heads, T, layout):
    announce(f"page append {heads} {T} {layout}")
    Hq, Hkv, D = heads
    s = Rows(T + D, T=T, Hq=Hq, Hkv=Hkv, D=D)
    s.check_read(s.check(*s.run(layout)))


@pytest.mark.parametrize("rotary", [0, 16, 48, 64, 128])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_part_of_a_head_turns(rotary, layout):
    announce(f"page append rotary {rotary} {layout}")
    s = Rows(3, T=3, D=128, Tp=70001)
    s.check(*s.run(layout, rotary, 5e5, 1.2, fused=True))


def test_ragged_counts_finished_cells_and_positions():
    announce("page append ragged")
    s = Rows(5, C=5, T=6, steps=[0, 63, -1, 130, 194], new=[6, 2, 6, 0, 6])
    pos = np.random.default_rng(1).integers(-9, 2**31, (5, 6))
    s.check_read(s.check(*s.run(pos=pos)))
    s = Rows(6, C=5, T=6, steps=[0, 63, -1, 130, 194], new=[6, 2, 6, 0, 6])
    s.check_read(s.check(*s.run()))


def test_many_cells():
    announce("page append 70 cells")
    s = Rows(7, C=70, T=2, Hq=2, Hkv=1, cap=66)
    s.check_read(s.check(*s.run()))


def test_absent_pages_drop_rows():
    announce("page append absent")
    s = Rows(8, C=3, T=70, steps=[0, 30, 100])
    s.tables[0, 0], s.tables[1, 1], s.tables[2, 2] = -1, s.n_pages, 2**31 - 1
    s.check_read(s.check(*s.run()))


def test_infinities_nan_zeros_and_far_sizes():
    announce("page append specials")
    s = Rows(9, C=2, T=8, Hq=4, Hkv=4, D=64, spread=0)
    s.k[0, 0, 0, 3], s.v[0, 1, 1, 40], s.k[0, 2, 2, 63] = float("inf"), float("nan"), float("-inf")
    s.k[0, 3], s.v[0, 4] = 0, 0
    s.k[0, 5] *= 1e-38
    s.v[0, 6] *= 2.0 ** -110
    s.v[0, 7, 0, :] = float(torch.finfo(torch.bfloat16).max)
    s.v[0, 7, 1, :32] = -2.0 ** 127 * 1.5
    s.v[1, 0] = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5] * 8, dtype=torch.bfloat16)   # ties
    s.v[1, 1] = torch.tensor([-6.03125, 12, -.25, .75, -1.25, 1.75, -2.5, 3.5] * 8, dtype=torch.bfloat16)
    s.q[1, 0, 0, 0] = float("nan")
    s.check_read(s.check(*s.run(rotary=0)))


def test_in_place_query_and_another_stream():
    announce("page append in place, stream")
    s = Rows(10, C=3, T=3)
    side = torch.cuda.Stream()
    s.check(*s.run(stream=side))
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    q = s.q.cuda()
    freq = up(s.freq)
    sp.splice_page_append(s.shape, s.pages, sp.make_rope("half", s.D), freq, s.steps, None, s.tab, q, s.k.cuda(), s.v.cuda(), q, s.mem)
    out, *want = s.run()
    assert torch.equal(out, q)


def test_rows_without_queries():
    announce("page append rows only")
    s = Rows(13, C=3, T=70)
    out, *want = s.run()
    full = s.mem.clone()
    s.mem.copy_(torch.from_numpy(s.pool.reshape(s.n_pages, -1)))
    freq = torch.from_numpy(s.freq).cuda()
    sp.splice_page_append(s.shape, s.pages, sp.make_rope("half", s.D), freq, s.steps, None, s.tab, None, s.k.cuda(), s.v.cuda(), None, s.mem)
    assert torch.equal(s.mem, full)


def test_replayed_graph():
    """A captured append and read keeps its steps, and takes what its tensors hold at each replay."""
    announce("page append graph")
    s = Rows(11, C=2, T=3, steps=[62, 5])
    s.run()
    q, k, v, out = s.q.cuda(), s.k.cuda(), s.v.cuda(), torch.zeros(2, 3, s.Hq, s.D, dtype=torch.bfloat16, device="cuda")
    rows = [torch.zeros(2, s.Hkv, 3, s.D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    freq, rope = torch.from_numpy(s.freq).cuda(), sp.make_rope("half", s.D)
    calls = lambda: (sp.splice_page_append(s.shape, s.pages, rope, freq, s.steps, None, s.tab, q, k, v, out, s.mem),  # noqa: E731
                     sp.splice_page_read(s.shape, s.pages, s.steps, None, s.tab, s.mem, *rows))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, *rows)]
        calls()
        torch.cuda.synchronize()
        for x, y in zip(got, (out, *rows)):
            assert torch.equal(x, y), i


def test_refused_tensors():
    announce("page append refusals")
    s = Rows(12)
    s.run()
    rope, f = sp.make_rope("half", 64), torch.zeros(32, dtype=torch.float64, device="cuda")
    q, k, v = s.q.cuda(), s.k.cuda(), s.v.cuda()
    out = torch.empty_like(q)
    call = lambda **kw: sp.splice_page_append(**{**dict(shape=s.shape, pages=s.pages, rope=rope, freq=f, cell_step=s.steps, cell_new=None,  # noqa: E731
                                                        tables=s.tab, q=q, k=k, v=v, q_out=out, pool=s.mem), **kw})
    for bad in (dict(q=s.q), dict(k=k.float()), dict(v=v[:, :, :1]), dict(tables=s.tab.long()), dict(tables=s.tab[:, :2]),
                dict(pool=s.mem[:-1]), dict(pool=s.mem.cpu()), dict(q_out=out.transpose(1, 2)), dict(freq=None), dict(cell_new=[1, 2]),
                dict(cell_step=s.steps[:2]), dict(q_out=None), dict(q=None)):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(sp.SpliceError):
        call(cell_new=[5, 0, 0])
    call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,mscale", [(64, 1.0), (128, 1.05), (256, 1.0)])
def test_rotated_keys_beyond_float32(D, mscale, layout):
    """Finite keys whose rotation passes the largest float stop at their largest code, as all above 3 * 2^126 do."""
    announce(f"page append far keys {D} {layout}")
    s = Rows(14, C=2, T=6, Hq=4, Hkv=2, D=D)
    top = float(torch.finfo(torch.bfloat16).max)
    sign = torch.sign(torch.randn(s.k.shape, generator=torch.Generator().manual_seed(D))).to(torch.bfloat16)
    s.k[0] = sign[0] * top
    s.k[1, 0, :, ::3] = sign[1, 0, :, ::3] * top
    s.k[0, 3, 0, 7], s.v[0, 4, 1, 5] = float("inf"), float("nan")
    out, q, k, v = s.run(layout, mscale=mscale)
    assert (np.abs(k[np.isfinite(k)]) > torch.finfo(torch.float32).max).any()
    s.check_read(s.check(out, q, k, v))
