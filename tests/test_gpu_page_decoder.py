"""A sweep decoded over 4-bit pages (SweepDecoder.make_pages, page_logits, PageCache): prompts quantised, a trunk decoded, cells
forked from it, ragged passes, rows dropped, against the float64 decode loop of oracle.decoder over the rows that the pages
hold."""
import numpy as np
import pytest
import torch

import decode_bar
import gpu_common as gc
import page_reference
import paper_2605_30574_amd as sp
import workloads
from oracle import decoder as ref
from paper_2605_30574_amd import decode
from test_gpu_tree_pass import TREE_REL
from workloads.model import make_weights

pytestmark = pytest.mark.gpu
STEPS = 140


class OverPages(ref.ReferenceDecoder):
    """The reference decoder, whose generated rows are those that the pages hold (checked here to be the step's, to a third of
    their block's largest value: half of the widest step between codes)."""
    rows = None    # [layer] (k, v) float64 [C][Hkv][STEPS][D]

    def attend(self, l, c, s, q_c):
        for cache, held in ((self.gen_k, self.rows[l][0]), (self.gen_v, self.rows[l][1])):
            want, got = ref.from_bf16_bits(cache[l][c, :, s]), held[c, :, s]
            top = np.repeat(np.abs(want.reshape(want.shape[0], -1, 32)).max(-1), 32, -1).reshape(want.shape)
            assert (np.abs(got - want) <= top / 3 * 1.05 + 1e-3).all(), (l, c, s)
            cache[l][c, :, s] = ref.to_bf16_bits(got)
        return super().attend(l, c, s, q_c)


def setup(name, dtype=torch.float32):
    w, m = decode_bar.case(name).with_(n_steps=STEPS), decode_bar.MODEL
    lw = workloads.cell_lw(w)
    wt = make_weights(w, m, dtype=dtype)
    on = lambda t: t.cuda()  # noqa: E731
    gpu_wt = {"embed": on(wt["embed"]), "lm_head": on(wt["lm_head"]), "norm_f": on(wt["norm_f"]),
              "layers": [{k: on(v) for k, v in L.items()} for L in wt["layers"]]}
    caches = [gc.gpu_layer(w, l, n_cells=lw.shape[0]) for l in range(w.n_layers)]
    prompts = []
    for c in caches:   # what the pages hold of them
        kept = {k: v for k, v in gc.host(c).items() if k in ("clean_k", "clean_v", "donor_k", "donor_v")}
        prompts.append({k: None if v is None else
                        ref.to_bf16_bits(page_reference.dequantised(*page_reference.quantised(ref.from_bf16_bits(v)))) for k, v in kept.items()})
    return w, m, lw, decode.SweepDecoder(w, m, gpu_wt, caches, lw), OverPages(w, m, decode_bar.f64_weights(wt), prompts, lw)


def held_rows(cache, count):
    """Rows 0 .. count[c] - 1 of every cell and layer, as the pages hold them."""
    sh = cache.shape
    got = []
    for l in range(sh.n_layers):
        rows = [torch.zeros(sh.n_cells, sh.n_kv_heads, STEPS, sh.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        sp.splice_page_read(sh, cache.pages(STEPS), np.zeros(sh.n_cells, np.int32), count, cache.tables, cache.pools[l], *rows)
        got.append([x.double().cpu().numpy() for x in rows])
    return got


def run(gpu, cpu, pages, tokens, steps, new, what):
    """One pass on both sides; every token's logits within the bar."""
    C, n = tokens.shape
    gc.announce(what)
    got = gpu.page_logits(torch.from_numpy(tokens).cuda(), pages, steps, new).double().cpu().numpy().reshape(C, n, -1)
    count = np.where(steps >= 0, n if new is None else new, 0)
    cpu.rows = held_rows(pages.cache, (np.maximum(steps, 0) + count).astype(np.int32))
    for t in range(n):
        at = np.where(t < count, steps + t, -1).astype(np.int32)
        want = cpu.forward(tokens[:, t], at)
        on = at >= 0
        if on.any():
            err = np.abs(got[on, t] - want[on]).max() / max(1.0, np.abs(want[on]).max())
            assert err <= TREE_REL, f"{what} token {t}: logits off by {err:.2e}"


@pytest.mark.parametrize("name", decode_bar.CASES)
def test_a_sweep_forked_from_its_trunk(name):
    w, m, lw, gpu, cpu = setup(name)
    C = lw.shape[0]
    rng = np.random.default_rng(3)
    draw = lambda n: rng.integers(0, m.vocab, (C, n))  # noqa: E731
    prompt = -(-w.prompt_len // 64)
    first = gpu.make_pages(50, n_pages=2 * prompt + 3 * C)
    cache = first.cache
    assert int(cache.missing) == 0
    only = lambda s: np.array([s] + [-1] * (C - 1), np.int32)  # noqa: E731
    # the trunk: 50 tokens in one pass, then 20, over two pages
    cache.reserve([50] + [0] * (C - 1))
    run(gpu, cpu, first, draw(50), only(0), None, f"{name} trunk")
    cache.reserve([70] + [0] * (C - 1))
    run(gpu, cpu, gpu.make_pages(20, cache=cache), draw(20), only(50), None, f"{name} trunk, on")
    # every cell from its row 70: the whole page is shared, the part of one copied
    before = held_rows(cache, np.array([70] + [0] * (C - 1)))
    cache.fork([0] * C, [70] * C, [75] * C)
    assert int(cache.missing) == 0
    after = held_rows(cache, np.full(C, 70))
    for (k, v), (k2, v2) in zip(before, after):
        assert all((k2[c, :, :70] == k[0, :, :70]).all() and (v2[c, :, :70] == v[0, :, :70]).all() for c in range(C))
    tables = cache.tables.cpu().numpy()
    assert len(set(tables[:, 0])) == 1 and len(set(tables[:, 1])) == C
    for rows in (cpu.gen_k, cpu.gen_v):
        for x in rows:
            x[1:] = x[0]
    new = np.arange(C, dtype=np.int32) % 6
    new[-1] = 5
    run(gpu, cpu, gpu.make_pages(5, cache=cache), draw(5), np.full(C, 70, np.int32), new, f"{name} forked")
    # of five tokens the first and the third stay; cells with fewer give theirs back, one is done
    whole = new == 5
    keep = np.full((C, 5), -1, np.int32)
    keep[whole, :2] = 0, 2
    cache.compact(np.full(C, 70, np.int32), torch.from_numpy(keep).cuda())
    rows = np.where(whole, 72, 70).astype(np.int32)
    parent = np.arange(C)
    parent[2], rows[2] = -1, 0
    cache.fork(parent, rows, np.where(parent >= 0, rows + 60, 0))
    assert int(cache.missing) == 0
    for x in (*cpu.gen_k, *cpu.gen_v):
        x[whole, :, 71] = x[whole, :, 72]
    steps = np.where(parent >= 0, rows, -1).astype(np.int32)
    run(gpu, cpu, gpu.make_pages(1, cache=cache), draw(1), steps, None, f"{name} kept")
    run(gpu, cpu, gpu.make_pages(59, cache=cache), draw(59), np.where(steps >= 0, steps + 1, -1).astype(np.int32), None, f"{name} far")


@pytest.mark.parametrize("dtype", [torch.bfloat16])
def test_bf16_weights_take_the_library_kernels(dtype):
    """A pass around bf16 weights: many tokens at once and one at a time say the same (each with its own roundings of the products:
    the bar of two passes)."""
    w, m, lw, gpu, _ = setup("blank-sink", dtype)
    C, n = lw.shape[0], 6
    tokens = torch.from_numpy(np.random.default_rng(9).integers(0, m.vocab, (C, n))).cuda()
    gc.announce("pages, bf16 weights")
    many, one = gpu.make_pages(n), gpu.make_pages(1)
    for p in (many, one):
        p.cache.reserve([n] * C)
    steps = np.zeros(C, np.int32)
    a = gpu.page_logits(tokens, many, steps).float().view(C, n, -1)
    for t in range(n):
        b = gpu.page_logits(tokens[:, t:t + 1].contiguous(), one, steps + t).float()
        # bf16 products and logits round at 2^-8 of their size in either pass, through two layers; a code next to a border may fall
        # on either side of it, a third of a row's largest value in one of 64 values
        assert (a[:, t] - b).abs().max() <= 0.1 * max(1.0, float(b.abs().max())), t


def test_replayed_pass():
    """A captured pass over pages: the rows it was captured for, with the tables and tokens of each replay."""
    w, m, lw, gpu, _ = setup("diff-G8", torch.bfloat16)
    C, n = lw.shape[0], 2
    pages = gpu.make_pages(n)
    pages.cache.reserve([64 + n] * C)
    rng = np.random.default_rng(11)
    tokens = torch.from_numpy(rng.integers(0, m.vocab, (C, n))).cuda()
    fill = gpu.make_pages(64, cache=pages.cache)
    gpu.page_logits(torch.from_numpy(rng.integers(0, m.vocab, (C, 64))).cuda(), fill, np.zeros(C, np.int32))
    steps = np.full(C, 64, np.int32)
    gc.announce("pages, graph")
    gpu.page_logits(tokens, pages, steps)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gpu.page_logits(tokens, pages, steps)
    for i in range(4):
        tokens.copy_(torch.from_numpy(rng.integers(0, m.vocab, (C, n))))
        pages.cache.fork(rng.permutation(C), [64] * C, [64 + n] * C)      # other cells' rows, other pages
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, gpu.page_logits(tokens, pages, steps)), i


def test_cache_refusals():
    w, m, lw, gpu, _ = setup("blank-sink")
    C = lw.shape[0]
    gc.announce("pages, refusals")
    pages = gpu.make_pages(2)
    cache = pages.cache
    for bad in (lambda: cache.reserve([STEPS + 1] * C), lambda: cache.reserve([1] * (C - 1)), lambda: cache.fork([0] * C, [5] * C),
                lambda: gpu.page_logits(torch.zeros(C, 3, dtype=torch.int64, device="cuda"), pages, np.zeros(C, np.int32)),
                lambda: cache.load_prompt(0, torch.zeros(1, 2, 3), torch.zeros(1, 2, 3)),
                lambda: sp.PageCache(255, 1, 4, 2, 64, 0, (0, 0), 64, 4)):
        with pytest.raises(ValueError):
            bad()
    zero = sp.PageCache(2, 1, 4, 2, 64, 64, (0, 64), 64, 4, donor_zero=True)
    rows = torch.zeros(2, 64, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: cache.fork([C] + [-1] * (C - 1), [0] * C),                     # a prompt is no cell
                lambda: sp.PageCache(2, 1, 4, 2, 64, 65, (0, 64), 64, 3),              # too few pages for the prompts
                lambda: zero.load_prompt(0, rows, rows, donor=True)):
        with pytest.raises(ValueError):
            bad()
    small = gpu.make_pages(1, n_pages=2 * (-(-w.prompt_len // 64)) + 1)
    small.cache.reserve([64] * C)
    assert int(small.cache.missing) == C - 1


def rounded(x):
    return ref.from_bf16_bits(ref.to_bf16_bits(x))


class RoundedOverPages(OverPages):
    """... whose products take and give bfloat16, as those of bfloat16 weights do; sums, norms and residuals stay float64."""

    def forward(self, tokens, steps):
        w, m, wt, C = self.w, self.m, self.wt, self.C
        heads = lambda x, n: x.reshape(C, n, w.head_dim)  # noqa: E731
        pos = w.prompt_len + np.maximum(steps, 0)
        x = wt["embed"][tokens]
        for l in range(self.N):
            p = wt["layers"][l]
            h = rounded(ref._rms_norm(x, p["norm_1"], m.rms_eps))
            q, k, v = (heads(rounded(h @ p[n]), e) for n, e in (("w_q", w.n_q_heads), ("w_k", w.n_kv_heads), ("w_v", w.n_kv_heads)))
            q, k, v = (ref.to_bf16_bits(y) for y in (ref._rope(q, pos, m.rope_theta), ref._rope(k, pos, m.rope_theta), v))
            o = np.zeros((C, w.n_q_heads, w.head_dim))
            for c in np.flatnonzero(steps >= 0):
                s = int(steps[c])
                self.gen_k[l][c, :, s], self.gen_v[l][c, :, s] = k[c], v[c]
                o[c] = rounded(self.attend(l, c, s, q[c]))
            x = x + rounded(o.reshape(C, -1) @ p["w_o"])
            h = rounded(ref._rms_norm(x, p["norm_2"], m.rms_eps))
            x = x + rounded(rounded(rounded(ref._silu(rounded(h @ p["w_gate"]))) * rounded(h @ p["w_up"])) @ p["w_down"])
        return rounded(rounded(ref._rms_norm(x, wt["norm_f"], m.rms_eps)) @ wt["lm_head"])


@pytest.mark.parametrize("name", decode_bar.CASES)
def test_bf16_weights_against_the_reference(name):
    """Passes of one and of many tokens around bfloat16 weights: off by the attention's own bar (TREE_REL less a rounding), and a
    logit by one step of bfloat16, 2^-7 at most, where the two sides round to its neighbours."""
    w, m, lw, gpu, cpu = setup(name, torch.bfloat16)
    cpu.__class__ = RoundedOverPages
    C, rng = lw.shape[0], np.random.default_rng(21)
    pages = gpu.make_pages(70)
    pages.cache.reserve([76] * C)
    for n, at in ((70, 0), (1, 70), (5, 71)):
        tokens = rng.integers(0, m.vocab, (C, n))
        gc.announce(f"{name} bf16 weights, {n} at {at}")
        p = gpu.make_pages(n, cache=pages.cache)
        got = gpu.page_logits(torch.from_numpy(tokens).cuda(), p, np.full(C, at, np.int32)).double().cpu().numpy().reshape(C, n, -1)
        cpu.rows = held_rows(pages.cache, np.full(C, at + n, np.int32))
        for t in range(n):
            want = cpu.forward(tokens[:, t], np.full(C, at + t, np.int32))
            err = np.abs(got[:, t] - want).max() / max(1.0, np.abs(want).max())
            assert err <= TREE_REL + 2.0 ** -8, f"{name} token {at + t}: logits off by {err:.2e}"
