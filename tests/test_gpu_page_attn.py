"""splice_page_attn against the definition in float64."""
import numpy as np
import pytest
import torch

import page_reference as ref
from page_common import RAGGED, SHARED, P, Sweep, announce, ragged_case, shared_case, sp

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (4, 4, 64), (8, 1, 128), (4, 2, 128), (2, 2, 256), (8, 2, 256)]


def run(s, split=0, what=""):
    announce("page attn " + what)
    s.check(*s.attend(split), what)


@pytest.mark.parametrize("T", [1, 2, 5, 17, 40])
@pytest.mark.parametrize("heads", HEADS)
def test_head_layouts_and_tokens(heads, T):
    Hq, Hkv, D = heads
    s = Sweep(100 + T, C=3, T=T, Hq=Hq, Hkv=Hkv, D=D, cap=T + 70)
    run(s, what=f"{heads} T={T}")


@pytest.mark.parametrize("Tp,span", [(0, (0, 0)), (1, (0, 1)), (1, (0, 0)), (63, (0, 63)), (64, (0, 64)), (65, (1, 64)),
                                     (129, (64, 64)), (300, (37, 290))])
@pytest.mark.parametrize("donor", ["diff", "zero"])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_and_spans(Tp, span, donor, D):
    s = Sweep(7, C=4, T=6, D=D, Tp=Tp, span=span, donor=donor, steps=[0, 5, -1, 60], LW=[[0, 0], [0, 7], [0, 0], [9, 0]])
    run(s, what=f"Tp={Tp} span={span} {donor} D={D}")


@pytest.mark.parametrize("window", [1, 2, 5, 63, 64, 65, 200])
@pytest.mark.parametrize("donor", ["diff", "zero"])
@pytest.mark.parametrize("T", [1, 12, 80])
def test_windows(window, donor, T):
    s = Sweep(11, C=4, T=T, Hq=4, Hkv=2, D=64, Tp=150, span=(20, 140), window=window, donor=donor, cap=T + 100, steps=[0, 3, 70, 98],
              LW=[[0, 0], [0, 7], [0, 75], [9, 0]])
    run(s, what=f"window={window} {donor} T={T}")


@pytest.mark.parametrize("onset", [0, 3, 10, 13, 16, 21, 22])
def test_onset_inside_the_tokens(onset):
    s = Sweep(13, C=2, T=12, D=128, Tp=100, span=(10, 95), steps=[10, 10], LW=[[0, onset], [2, 0]])
    run(s, what=f"onset={onset}")


@pytest.mark.parametrize("split", [64, 128, 256, 1024])
@pytest.mark.parametrize("T,D", [(1, 64), (2, 128), (12, 128), (40, 128), (10, 256)])
def test_splits(T, D, split):
    s = Sweep(17, C=3, T=T, Hq=4, Hkv=2, D=D, Tp=700, span=(100, 620), cap=T + 500, steps=[0, 77, 500], LW=[[0, 0], [0, 80], [9, 0]])
    run(s, split, f"split={split} T={T} D={D}")


@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("donor,window", [("diff", 0), ("zero", 0), ("diff", 1500), ("zero", 500)])
def test_a_prompt_shared_by_many_cells(T, D, donor, window):
    """Tiles of several cells' rows over the prompt: enough cells and slots for the plan to take them."""
    C = 16 if D == 128 else (30 if D == 64 else 9)
    steps = np.random.default_rng(3).integers(0, 70, C)
    steps[5] = -1
    LW = [[0, 0] if c % 3 == 0 else ([9, 0] if c % 3 == 1 else [1, int(steps[c]) + 1]) for c in range(C)]
    s = Sweep(23, C=C, T=T, Hq=8, Hkv=2, D=D, Tp=1500, span=(70, 1300), donor=donor, window=window, cap=80, steps=steps, LW=LW)
    run(s, what=f"shared T={T} D={D} {donor} {window}")


@pytest.mark.parametrize("kind,case", [(kind, case) for kind in SHARED for case in SHARED[kind]])
def test_tiles_of_several_cells(kind, case):
    """test_page_plan.py holds that the plan takes them for these shapes."""
    s = Sweep(97, donor=kind[0], window=kind[1], **shared_case(*case))
    s.tables[3, 0] = -1
    run(s, what=f"several cells {kind} {case}")


def test_tiles_of_several_cells_in_other_parts():
    s = Sweep(98, **shared_case(*SHARED["diff", 0][2]))
    for split in (64, 512, 65536):
        run(s, split, f"several cells, parts of {split}")


def test_ragged_tokens():
    s = Sweep(29, C=6, T=33, Hq=4, Hkv=2, D=64, Tp=70, span=(3, 60), cap=130, steps=[0, 10, 60, -1, 97, 100], new=[33, 0, 1, 33, 33, 17])
    run(s, what="ragged")
    s = Sweep(30, C=40, T=4, Hq=8, Hkv=1, D=64, Tp=30, span=(3, 20), cap=66, new=np.arange(40) % 5)
    run(s, what="ragged, many cells")


def test_one_cell_many_keys():
    s = Sweep(31, C=1, T=1, Hq=8, Hkv=2, D=128, Tp=5000, span=(100, 4900), cap=3000, steps=[2999], LW=[[0, 10]])
    run(s, what="one cell, many keys")


@pytest.mark.parametrize("D,T", [(64, 300), (128, 200), (256, 150)])
def test_a_prompts_own_pass(D, T):
    s = Sweep(37, C=2, T=T, Hq=4, Hkv=1, D=D, Tp=0, span=(0, 0), cap=T + 30, steps=[0, 30], new=[T, T - 7])
    run(s, what=f"prompt D={D}")


def test_shared_pages():
    """Cells that name the same pages, and a page named twice by one table."""
    s = Sweep(41, C=4, T=2, Hq=4, Hkv=2, D=64, cap=300, steps=[298, 200, 150, 130])
    s.tables[1:, :2] = s.tables[0, :2]
    s.tables[2, 1] = s.tables[2, 0]
    s.clean[:] = s.tables[0, :1]
    run(s, what="shared pages")


@pytest.mark.parametrize("T", [1, 40])
def test_absent_pages_are_seen_by_nobody(T):
    s = Sweep(43, C=3, T=T, Hq=4, Hkv=2, D=64, Tp=200, span=(50, 150), cap=300, steps=[250, 100, 10], LW=[[0, 0], [9, 0], [0, 0]])
    s.tables[0, 1], s.tables[0, 2], s.tables[1, 0], s.clean[1], s.donor[2] = -1, s.n_pages, -2**31, 2**31 - 1, -1
    run(s, what="absent")


def test_nothing_to_see():
    s = Sweep(47, C=2, T=2, Hq=4, Hkv=2, D=64, Tp=70, span=(0, 0), cap=100, steps=[20, 90])
    s.tables[:], s.clean[:], s.donor[:] = -1, -1, s.n_pages
    announce("page attn nothing")
    out, lse = s.attend()
    assert (out == 0).all() and (lse == -float("inf")).all()
    s = Sweep(48, C=2, T=1, Hq=4, Hkv=2, D=64, Tp=0, span=(0, 0), cap=100, steps=[20, 90], window=1)
    s.tables[0] = -1
    run(s, what="nothing for one cell")


@pytest.mark.parametrize("T", [1, 9, 70])
def test_nan_rows_reach_only_who_sees_them(T):
    """Stored infinities and NaN: bytes 255.  Tokens before such a row, and other heads, are what they would be."""
    s = Sweep(53, C=3, T=T, Hq=4, Hkv=2, D=64, Tp=100, span=(20, 90), cap=T + 80, steps=[10, 60, 70], LW=[[0, 0], [9, 0], [0, 0]])
    def spoil(page, r, h):
        _, _, ks, vs = ref.places(r, np.arange(s.D), s.D)
        s.pool[page, h, ks], s.pool[page, h, vs] = 255, 255
    spoil(s.clean[0], 30, 0)                                  # seen by unspliced tokens only
    for c in (0, 1):
        r = int(s.steps[c]) + T // 2                          # a new token in the middle
        spoil(s.tables[c, r // P], r % P, 1)
    announce(f"page attn nan T={T}")
    out, lse = s.attend()
    s.check(out, lse)
    assert torch.isnan(lse).any() and not torch.isnan(lse).all()


def test_queries_with_infinities_nan_and_far_sizes():
    s = Sweep(59, C=2, T=3, Hq=4, Hkv=2, D=128, cap=90)
    s.q[0, 0, 0, 5], s.q[0, 1, 1, 127], s.q[1, 0, 2, 0] = float("inf"), float("nan"), -float("inf")
    s.q[0, 2, 0] = 0
    s.q[0, 2, 1] *= 2.0 ** -100
    s.q[0, 2, 2, 7] = 300.0                                   # one large value among small ones
    s.q[1, 1, 3] *= 40
    announce("page attn specials")
    out, lse = s.attend()
    bad = torch.zeros(2, 3, 4, dtype=torch.bool)
    bad[0, 0, 0] = bad[0, 1, 1] = bad[1, 0, 2] = True
    assert (torch.isnan(lse.cpu()) == bad).all() and (torch.isnan(out.cpu()).all(-1) == bad).all()
    for i in np.argwhere(bad.numpy()):
        s.q[tuple(i)] = 0
        out[tuple(i)], lse[tuple(i)] = 0, 0
    wo, wl, to, tl = s.expected()
    ok = ~bad.numpy()
    assert (np.abs(out.double().cpu().numpy() - wo)[ok] <= to[ok]).all() and (np.abs(lse.double().cpu().numpy() - wl)[ok] <= tl[ok]).all()


def test_values_of_far_exponents():
    s = Sweep(61, C=2, T=2, Hq=4, Hkv=2, D=64, Tp=40, cap=90, spread=30)
    run(s, what="far exponents")


def test_a_running_maximum_that_climbs():
    """Scores that rise by more than 2^8 from page to page, and an outlier at the first key."""
    s = Sweep(67, C=1, T=1, Hq=4, Hkv=1, D=64, Tp=0, span=(0, 0), cap=900, steps=[899])
    direction = s.q[0, 0, 0].double().numpy()
    for j in range(s.L):
        k = np.tile(direction * 0.35 * (j + 1), (P, 1)) + 0.05 * s.rng.standard_normal((P, s.D))
        s.put(s.tables[0, j], 0, k, s.rng.standard_normal((P, s.D)), range(P))
    run(s, what="climbing")
    run(s, 64, "climbing, split")


def test_a_pool_beyond_32_bits():
    """Offsets that pass 32 bits: the pages in use are the last ones of a pool of 4.6 GB."""
    s = Sweep(71, C=2, T=2, Hq=4, Hkv=2, D=256, Tp=70, span=(3, 60), cap=100)
    far = 130000
    announce("page attn far pool")
    s.send()
    big = torch.zeros(far + s.n_pages, s.pool[0].size, dtype=torch.uint8, device="cuda")
    big[far:] = s.dev["pool"]
    want = s.attend(send=False)
    s.pages.n_pages = far + s.n_pages
    s.dev.update(pool=big, **{k: s.dev[k] + far for k in ("tables", "clean", "donor")})
    got = s.attend(send=False)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_same_bits_twice_and_a_workspace_of_garbage():
    s = Sweep(73, C=3, T=1, Hq=8, Hkv=2, D=128, Tp=2000, span=(100, 1900), cap=500)
    announce("page attn bits")
    want = s.attend()
    ws = torch.full((sp.splice_page_attn_workspace_bytes(s.shape, s.call, s.pages),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        got = s.attend(ws=ws, send=False)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s.check(*want)


def test_replayed_graph_and_another_stream():
    s = Sweep(79, C=3, T=2, Hq=8, Hkv=2, D=128, Tp=1500, span=(100, 1400), cap=300)
    announce("page attn graph")
    s.check(*s.attend(stream=torch.cuda.Stream()))
    d = s.dev
    out, lse = torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 2, 8, device="cuda")
    ws = torch.empty(sp.splice_page_attn_workspace_bytes(s.shape, s.call, s.pages), dtype=torch.uint8, device="cuda")
    call = lambda: sp.splice_page_attn(s.shape, s.call, s.pages, s.LW, s.steps, None, d["tables"], d["clean"], d["donor"], d["q"],  # noqa: E731
                                       d["pool"], out, lse, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        d["q"].normal_()
        d["tables"].copy_(d["tables"][torch.randperm(3, device="cuda")])   # other pages: all hold rows
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        call()
        torch.cuda.synchronize()
        # by their bits: a cell may now see rows that are none of its own, NaN among them
        assert torch.equal(got[0].view(torch.int16), out.view(torch.int16)) and torch.equal(got[1].view(torch.int32), lse.view(torch.int32)), i


def test_refused_tensors():
    s = Sweep(83)
    announce("page attn refusals")
    s.attend()
    d = s.dev
    out, lse = torch.empty(3, 1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 1, 8, device="cuda")
    ws = torch.empty(sp.splice_page_attn_workspace_bytes(s.shape, s.call, s.pages), dtype=torch.uint8, device="cuda")
    good = dict(shape=s.shape, call=s.call, pages=s.pages, cell_LW=s.LW, cell_step=s.steps, cell_new=None, tables=d["tables"],
                clean_table=d["clean"], donor_table=d["donor"], q=d["q"], pool=d["pool"], out=out, lse=lse, workspace=ws)
    for bad in (dict(q=s.q), dict(q=d["q"].float()), dict(out=out.float()), dict(lse=lse[:1]), dict(tables=d["tables"].long()),
                dict(clean_table=None), dict(donor_table=None), dict(clean_table=d["clean"][:0]), dict(pool=d["pool"][:-1]),
                dict(cell_LW=s.LW[:1]), dict(cell_new=[1]), dict(lse=lse.cpu())):
        with pytest.raises(ValueError):
            sp.splice_page_attn(**{**good, **bad})
    for bad in (dict(cell_new=[2, 0, 0]), dict(cell_step=[100, 0, 0])):
        with pytest.raises(sp.SpliceError):
            sp.splice_page_attn(**{**good, **bad})
    sp.splice_page_attn(**good)
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,parts", [(64, 33), (64, 34), (64, 35), (128, 17), (128, 33), (128, 49)])
def test_numbers_of_parts_that_end_within_a_load(D, parts):
    """A wave of the join loads 256 / D parts at a time: the last load has fewer."""
    s = Sweep(43, C=1, T=300, Hq=4, Hkv=2, D=D, Tp=0, span=(0, 0), cap=parts * 64, steps=[parts * 64 - 300], LW=[[0, 0]])
    run(s, 64, f"D={D} {parts} parts")


@pytest.mark.parametrize("T,D", [(1, 64), (3, 128), (40, 128), (2, 256)])
def test_a_query_does_not_move_its_neighbours(T, D):
    """Queries of one tile do not share a running maximum: the others' bits stay where one of them is 100 times as large, or NaN."""
    s = Sweep(47, C=2, T=T, Hq=8, Hkv=2, D=D, Tp=150, span=(20, 140), cap=T + 300, steps=[200, 299])
    announce(f"neighbours T={T} D={D}")
    want, mine = s.attend(), s.q.clone()
    for other in (100.0, float("nan")):
        s.q = mine.clone()
        s.q[:, 0, 1] = s.q[:, 0, 1] * other
        got = s.attend()
        for x, y in zip(want, got):
            a, b = x.clone(), y.clone()
            a[:, 0, 1] = b[:, 0, 1] = 0
            assert torch.equal(a, b)


@pytest.mark.parametrize("case", RAGGED)
def test_tiles_of_several_cells_some_of_them_finished(case):
    """test_page_plan.py holds that the plan takes them for these shapes: a cell's number is not its place among those with tokens."""
    s = Sweep(101, **ragged_case(*case))
    s.tables[2, 0] = -1
    run(s, what=f"several cells, ragged {case}")


@pytest.mark.parametrize("split", [0, 256])
@pytest.mark.parametrize("T", [1, 3, 9, 40, 90])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_nan_rows_inside_of_runs(D, T, split):
    """Rows that are NaN in full pages of the prompt, the donor and a cell's rows, for each kind of work group and part."""
    s = Sweep(103, C=3, T=T, Hq=8, Hkv=2, D=D, Tp=700, span=(130, 600), cap=T + 500, steps=[499, 300, 20], LW=[[0, 0], [9, 0], [0, 20 + T // 2]])

    def spoil(page, r, h):
        _, _, ks, vs = ref.places(r, np.arange(s.D), s.D)
        s.pool[page, h, ks], s.pool[page, h, vs] = 255, 255
    spoil(s.clean[5], 17, 0)                                  # of the span: seen by unspliced tokens only
    spoil(s.donor[4], 63, 1)                                  # ... by spliced ones
    spoil(s.tables[0, 3], 0, 1)
    r = 300 + T // 2                                          # a new token in the middle
    spoil(s.tables[1, r // P], r % P, 1)
    announce(f"page attn nan inside D={D} T={T} split={split}")
    out, lse = s.attend(split)
    s.check(out, lse)
    assert torch.isnan(lse).any() and not torch.isnan(lse).all()


@pytest.mark.parametrize("case", [RAGGED[0], RAGGED[1], RAGGED[4]])
def test_nan_rows_in_a_shared_prompt(case):
    s = Sweep(107, **ragged_case(*case))
    for page, r, h in ((s.clean[9], 40, 0), (s.donor[7], 1, 1)):
        _, _, ks, vs = ref.places(r, np.arange(s.D), s.D)
        s.pool[page, h, ks], s.pool[page, h, vs] = 255, 255
    announce(f"page attn nan shared {case}")
    out, lse = s.attend()
    s.check(out, lse)
    assert torch.isnan(lse).any() and not torch.isnan(lse).all()
