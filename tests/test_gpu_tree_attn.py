"""splice_tree_attn against the definition in float64."""
import numpy as np
import pytest
import torch

from tree_common import Sweep, announce, f64, sp

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (4, 4, 64), (8, 1, 128), (4, 2, 128), (2, 2, 256), (8, 2, 256)]


def run(s, split=0, what=""):
    announce(what)
    s.check(*s.attend(split), what)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("T", [1, 3, 9, 17, 64])
@pytest.mark.parametrize("heads", HEADS)
def test_head_layouts_and_tree_sizes(heads, T, kv):
    Hq, Hkv, D = heads
    s = Sweep(100 + T, C=3, T=T, Hq=Hq, Hkv=Hkv, D=D, cap=T + 21, kv=kv)
    run(s, what=f"{heads} T={T} {kv}")


@pytest.mark.parametrize("Tp,span", [(0, (0, 0)), (1, (0, 1)), (1, (0, 0)), (31, (0, 31)), (64, (0, 64)), (65, (1, 64)),
                                     (129, (64, 64)), (300, (37, 290))])
@pytest.mark.parametrize("donor", ["diff", "zero"])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_and_spans(Tp, span, donor, D):
    s = Sweep(7, C=4, T=6, D=D, Tp=Tp, span=span, donor=donor, steps=[0, 5, -1, 20], LW=[[0, 0], [0, 7], [0, 0], [9, 0]])
    run(s, what=f"Tp={Tp} span={span} {donor}")


@pytest.mark.parametrize("window", [1, 2, 5, 30, 33, 200])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("donor", ["diff", "zero"])
def test_windows(window, kv, donor):
    chain = np.tile(np.arange(-1, 11), (4, 1))
    s = Sweep(11, C=4, T=12, D=64, Tp=70, span=(20, 66), window=window, kv=kv, donor=donor, steps=[0, 3, 9, 28],
              LW=[[0, 0], [0, 7], [0, 13], [9, 0]], parents=chain)
    run(s, what=f"window={window} {kv} {donor}")


@pytest.mark.parametrize("onset", [0, 3, 10, 13, 16, 21, 22])
def test_onset_inside_the_tree(onset):
    chain = np.tile(np.arange(-1, 11), (2, 1))
    s = Sweep(13, C=2, T=12, D=128, Tp=100, span=(10, 95), steps=[10, 10], LW=[[0, onset], [2, 0]], parents=chain)
    run(s, what=f"onset={onset}")


@pytest.mark.parametrize("split", [64, 128, 256, 1024])
@pytest.mark.parametrize("T,D", [(2, 64), (12, 128), (40, 128), (10, 256)])
def test_splits(T, D, split):
    s = Sweep(17, C=3, T=T, D=D, Tp=700, span=(100, 620), cap=T + 500, steps=[0, 77, 500], LW=[[0, 0], [0, 80], [9, 0]])
    run(s, split, f"split={split} T={T} D={D}")


def test_defaults_split_one_cell():
    s = Sweep(19, C=1, T=33, Hq=8, Hkv=2, D=128, Tp=2500, span=(100, 2400), cap=1200, steps=[1100], LW=[[0, 1110]])
    run(s, what="one cell, long prompt")


def test_any_word_is_a_mask():
    """Words that are no ancestors: some without the node itself, some empty, bits beyond T."""
    s = Sweep(23, C=5, T=20, Tp=0, span=(0, 0), steps=[0, 0, 3, 0, 9])
    rng = np.random.default_rng(1)
    s.visible[:] = rng.integers(0, 1 << 63, s.visible.shape, dtype=np.uint64)
    s.visible[0] = 0
    s.visible[3, ::2] = 0
    s.depth[1, 4] = 1000   # counts as T - 1
    s.send_tree()
    run(s, what="random words")


def test_nothing_visible_anywhere():
    s = Sweep(29, C=2, T=4, Tp=9, span=(0, 9), window=1, steps=[6, 2])
    s.visible[:] = 0
    s.send_tree()
    run(s, what="window 1, nodes that do not see themselves")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,D", [(7, 64), (20, 128), (40, 128), (9, 256)])
def test_what_is_not_seen_may_hold_anything(kv, T, D):
    """NaN and infinities in padding, in rows behind the tree, below a window, in the span of the other class and in nodes
    that a node does not see."""
    C = 3
    parents = np.full((C, T), -1)
    parents[:, 1:] = 0
    parents[1, T - 1] = -2
    s = Sweep(31, C=C, T=T, D=D, Tp=80, span=(16, 70), kv=kv, steps=[4, 9, 30], cap=30 + T + 3, LW=[[0, 0], [0, 0], [0, 0]],
              window=60, parents=parents)
    want = s.expected()
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), 3.0e38], dtype=torch.bfloat16, device="cuda")
    for x in s.clean:   # every cell is spliced: nobody reads the clean span
        x[:, 16:70, :4] = bad
    for c in range(C):
        n = int(s.steps[c])
        for x in s.gen:
            x[c, :, n + T:] = 0x7f if kv == "e4m3" else float("nan")
    for x in s.gen:
        x[1, :, 9 + T - 1] = 0x7f if kv == "e4m3" else float("inf")
    got = s.attend()
    s.expected = lambda: want
    s.check(*got, "NaN where nothing looks")
    # node 2 of cell 0 holds NaN and infinities: only node 2 sees it
    for x in s.gen:
        x[0, :, 4 + 2, :4] = 0x7f if kv == "e4m3" else bad
    out, lse = s.attend()
    torch.cuda.synchronize()
    o = f64(out)
    assert np.isnan(o[0, 2]).any()
    o[0, 2] = want[0][0, 2]
    l = f64(lse)
    l[0, 2] = want[1][0, 2]
    s.check(torch.from_numpy(o), torch.from_numpy(l), "NaN in a node that others do not see")


def test_infinite_values_that_are_seen():
    s = Sweep(37, C=1, T=3, D=64, Tp=5, span=(0, 0), steps=[2], parents=np.array([[-1, 0, 0]]))
    s.gen[1][0, :, 3, 0] = float("inf")    # node 1, seen by itself
    s.gen[1][0, :, 3, 1] = float("-inf")
    s.gen[1][0, :, 3, 2] = float("nan")
    out, _ = s.attend()
    torch.cuda.synchronize()
    o = f64(out)[0]
    assert (o[1, :, 0] == np.inf).all() and (o[1, :, 1] == -np.inf).all() and np.isnan(o[1, :, 2]).all()
    assert np.isfinite(o[[0, 2]]).all() and np.isfinite(o[1, :, 3:]).all()


def test_8_bit_cache_is_the_bf16_cache_of_its_values():
    s = Sweep(41, C=3, T=9, D=128, Tp=90, span=(10, 80), cap=300, kv="e4m3", steps=[0, 150, 291])
    out, lse = s.attend(128)
    b = Sweep(41, C=3, T=9, D=128, Tp=90, span=(10, 80), cap=300, steps=[0, 150, 291])
    for x in ("q", "clean", "donor", "depth_dev", "visible_dev", "LW"):
        setattr(b, x, getattr(s, x))
    b.gen = [torch.from_numpy(x).to(torch.bfloat16).cuda() for x in s.gen_values()]
    out_b, lse_b = b.attend(128)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), out_b.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse_b.view(torch.int32))


def test_single_chain_node_is_the_decode_step():
    """T = 1: what splice_decode_step computes, up to both kernels' roundings."""
    s = Sweep(43, C=6, T=1, Hq=8, Hkv=2, D=128, Tp=200, span=(20, 190), cap=90, steps=[0, 3, 50, -1, 89, 10])
    out, lse = s.attend()
    o2 = torch.full((6, 8, 128), 7.0, device="cuda")
    l2 = torch.full((6, 8), 7.0, device="cuda")
    at = torch.from_numpy(np.maximum(s.steps, 0)).long().cuda()
    new = [x[torch.arange(6, device="cuda"), :, at].contiguous() for x in s.gen]
    sp.splice_decode_step(s.shape, s.call(), s.LW, s.steps, s.q, *new, *s.clean, *s.donor, *s.gen, o2, l2, sp.new_workspace(s.shape))
    torch.cuda.synchronize()
    _, _, spread, _, _ = s.expected()
    spread = np.nan_to_num(spread[:, 0])
    assert (np.abs(f64(out)[:, 0] - f64(o2)) <= 2.0 ** -6 * spread + 1e-6).all()   # two roundings of P and one each of the results
    assert (np.abs(f64(lse)[:, 0] - f64(l2)) <= 1e-4).all()


def test_same_bits_again_and_on_another_stream():
    s = Sweep(47, C=4, T=10, D=128, Tp=600, span=(50, 500), cap=400)
    a = s.attend(128)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = s.attend(128, stream=other)
    other.synchronize()
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32),
                           y.view(torch.int16 if y.dtype is torch.bfloat16 else torch.int32))


def test_captured_and_replayed_on_new_inputs():
    s = Sweep(53, C=3, T=8, D=64, Tp=500, span=(50, 400), cap=300, steps=[100, 200, 290])
    out, lse = s.outputs()
    ws = s.workspace(256)
    s.attend(256, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.attend(256, out, lse, ws)
    for n in range(3):
        s.q.copy_(torch.randn(s.q.shape, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16))
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = s.attend(256)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        s.check(out, lse, f"replay {n}")


def test_cells_of_nothing():
    s = Sweep(59, C=3, T=4, steps=[-1, -5, -1])
    run(s, what="every cell finished")


def test_far_rows_of_a_large_cache():
    """Rows beyond 2^31 bytes of one cache tensor."""
    C, T, D, cap = 3, 3, 256, 1 << 20
    s = Sweep(61, C=C, T=T, Hq=2, Hkv=1, D=D, Tp=8, span=(0, 8), cap=64, steps=[40, 60, 61])
    big = []
    for x in s.gen:
        y = torch.empty(C, 1, cap * 2, D, dtype=torch.bfloat16, device="cuda")   # 3 GiB each
        y[:, :, :64] = x
        big.append(y)
    want = s.expected()
    small, s.gen, s.cap = s.gen, big, cap * 2
    s.shape = sp.make_shape(C, 4, 2, 1, D, 8, (0, 8), cap * 2, False, "bf16")
    got = s.attend(64)
    s.expected = lambda: want
    s.check(*got, "far rows")


# ---------------------------------------------------------------- many cells over one prompt

def many(seed, C, T, Tp=400, window=0, **kw):
    """Cells of every class: never spliced, from their first step on, from a depth within the tree on; some finished."""
    rng = np.random.default_rng(seed)
    cap = T + 60
    steps = rng.integers(0, cap - T + 1, C)
    if C > 4:
        steps[C // 2] = -1
    LW = [[9, 0] if c % 3 == 0 else ([0, 0] if c % 3 == 1 else [1, max(int(steps[c]), 0) + 1 + c % 2]) for c in range(C)]
    span = kw.pop("span", (Tp // 5, Tp - Tp // 7))
    return Sweep(seed, C=C, T=T, Tp=Tp, span=span, cap=cap, steps=steps, LW=LW, window=window, **kw)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads", [(8, 2, 64), (2, 2, 64), (8, 1, 128), (8, 2, 128), (8, 4, 256)])
@pytest.mark.parametrize("C,T", [(17, 1), (40, 2), (12, 5), (9, 16), (2, 16)])
def test_shared_prompt(C, T, heads, kv):
    """split_keys has the cells share the prompt's tiles at any size."""
    Hq, Hkv, D = heads
    s = many(200 + C + T, C, T, Hq=Hq, Hkv=Hkv, D=D, kv=kv)
    run(s, 256, f"shared prompt {C} {T} {heads} {kv}")
    run(s, what=f"apart {C} {T} {heads} {kv}")


@pytest.mark.parametrize("window", [1, 20, 64, 130, 300, 470])
@pytest.mark.parametrize("donor", ["diff", "zero"])
def test_shared_prompt_windows(window, donor):
    run(many(211, 14, 6, window=window, donor=donor, D=128), 256, f"shared prompt, window {window} {donor}")


@pytest.mark.parametrize("span", [(0, 400), (0, 0), (1, 399), (64, 128), (399, 400)])
@pytest.mark.parametrize("donor", ["diff", "zero"])
def test_shared_prompt_spans(span, donor):
    run(many(223, 11, 7, span=span, donor=donor, D=64), 256, f"shared prompt, span {span} {donor}")


@pytest.mark.parametrize("split", [64, 128, 1024])
def test_shared_prompt_splits(split):
    run(many(227, 13, 9, Tp=1100, D=128), split, what=f"shared prompt, split {split}")


@pytest.mark.parametrize("D", [64, 128, 256])
def test_shared_prompt_hides_what_is_not_seen(D):
    """NaN and infinities in the clean span, which only unspliced nodes see, and in the donor's outside of the span."""
    s = many(229, 12, 5, D=D, Hkv=4, window=450)
    want = s.expected()
    a, b = s.span
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), 3.0e38], dtype=torch.bfloat16, device="cuda")
    for x in s.donor:
        x[:, :a] = float("nan")
        x[:, b:, :4] = bad
    s.expected = lambda: want
    s.check(*s.attend(256), "NaN in the donor's scaffold")
    for x in s.clean:
        x[:, a + 3:b - 5, :4] = bad
    out, lse = s.attend(256)
    torch.cuda.synchronize()
    step = s.steps[:, None] + s.depth
    on = (s.depth >= 0) & (s.steps[:, None] >= 0)
    spliced = on & (s.layer >= s.LW[:, :1]) & (step >= s.LW[:, 1:])
    assert (spliced.any(1) & (on & ~spliced).any(1)).any()
    o, l = f64(out), f64(lse)
    assert not np.isfinite(o[on & ~spliced]).all(-1).any()
    o[on & ~spliced], l[on & ~spliced] = want[0][on & ~spliced], want[1][on & ~spliced]
    s.check(torch.from_numpy(o), torch.from_numpy(l), "NaN in the clean span")


def test_shared_prompt_of_every_cell():
    """As many cells as a call takes, one node each, and cells of one tile of rows that are all finished."""
    C = 256
    s = many(233, C, 1, Hq=4, Hkv=1, D=64, Tp=300)
    s.steps[32:64] = -1
    run(s, 256, "256 cells")
    run(s, what="256 cells apart")


def test_shared_prompt_by_default():
    run(many(241, 64, 2, Hq=2, Hkv=1, Tp=1400, D=64), what="64 cells over 1400 slots")


def test_large_values_keep_their_scale():
    """Values far beyond fp16's range go through the partial results by a power of two."""
    s = Sweep(239, C=2, T=9, D=128, Tp=900, span=(100, 800), cap=600, steps=[500, 20], LW=[[0, 0], [9, 0]])
    out, lse = s.attend(128)
    for x in (s.clean[1], s.donor[1], s.gen[1]):
        x.mul_(2.0 ** 100)
    big, lse2 = s.attend(128)
    torch.cuda.synchronize()
    assert torch.equal(lse, lse2)
    on = torch.from_numpy(s.depth >= 0).cuda()
    # the scaled partial results are rounded alike up to fp16's subnormals, the result after it
    got, want = big[on].double() * 2.0 ** -100, out[on].double()
    assert ((got - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -14).all()


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -50, 2.0 ** -100])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("T,D", [(2, 64), (9, 128), (12, 256)])
def test_small_values_keep_their_scale(T, D, shared, size):
    """Values far below fp16's range go through the partial results by a power of two of up to 2^60: at least ten bits of a
    row's largest value are left at 2^-60, and with it at 2^-100 the absolute error is 2^-25 2^-60."""
    s = Sweep(251, C=6 if shared else 2, T=T, D=D, Hq=4, Hkv=1, Tp=900, span=(100, 800), cap=600)
    for x in (s.clean[1], s.donor[1], s.gen[1]):
        x.mul_(size)
    out, lse = s.attend(128)
    if size >= 2.0 ** -50:
        s.check(out, lse, f"values of {size}")
    else:
        torch.cuda.synchronize()
        want = s.expected()[0]
        on = s.depth >= 0
        assert np.abs(f64(out) - want)[on].max() <= 2.0 ** -85


def test_no_cells():
    """A call of no cells checks its tensors and returns."""
    s = Sweep(257, C=0, T=3)
    out, lse = s.attend()
    rope = sp.make_rope("half", 64)
    freq = torch.ones(32, dtype=torch.float64, device="cuda")
    k = torch.empty(0, 3, s.Hkv, s.D, dtype=torch.bfloat16, device="cuda")
    sp.splice_tree_append(s.shape, s.tree, rope, freq, s.steps, s.depth_dev, s.q, k, k, out, *s.gen)
    sp.splice_tree_keep(s.shape, s.tree, s.steps, s.depth_dev, *s.gen)
    rows = torch.empty(0, s.Hkv, 3, s.D, dtype=torch.bfloat16, device="cuda")
    sp.splice_tree_read(s.shape, s.tree, s.steps, *s.gen, None, None, rows, rows.clone())
    torch.cuda.synchronize()


def test_two_calls_at_once():
    """Calls with workspaces of their own, on two streams at the same time, do not touch each other."""
    a, b = Sweep(263, C=3, T=9, D=128, Tp=900, span=(100, 800), cap=600), many(269, 40, 2)
    alone = [a.attend(128), b.attend(256)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    held = [[(s.outputs(), s.workspace(split)) for _ in range(8)] for s, split in ((a, 128), (b, 256))]
    torch.cuda.synchronize()
    for n in range(8):
        for s, split, stream, h in zip((a, b), (128, 256), streams, held):
            (out, lse), ws = h[n]
            s.attend(split, out, lse, ws, stream)
    torch.cuda.synchronize()
    for (out, lse), h in zip(alone, held):
        for (o, l), _ in h:
            assert torch.equal(o, out) and torch.equal(l, lse)


@pytest.mark.parametrize("split", [0, 64, 256])
@pytest.mark.parametrize("span", [(0, 1400), (3, 1390)])
@pytest.mark.parametrize("unspliced", [0, 1, 20, 39])
def test_zero_donor_whose_span_is_the_prompt(unspliced, span, split):
    """Cells that walk the whole prompt beside cells that walk nothing of it, or next to nothing."""
    C, T = 40, 5
    rng = np.random.default_rng(unspliced)
    steps = rng.integers(0, 60, C)
    steps[7] = -1
    LW = [[9, 0] if c < unspliced else [0, 0] for c in range(C)]
    if unspliced == 20:
        LW[19] = [0, max(int(steps[19]), 0) + 2]   # one on both sides of its onset
    s = Sweep(271, C=C, T=T, Tp=1400, span=span, cap=70, steps=steps, LW=LW, donor="zero", Hq=4, Hkv=1, D=128)
    run(s, split, f"ZERO donor, {unspliced} unspliced, span {span}, split {split}")
