"""A pass over trees of candidate tokens (SweepDecoder.score_tree, keep_nodes) against the float64 decode loop of
oracle.decoder, token by token, and against the plain decode loop that it stands for."""
import numpy as np
import pytest
import torch

import decode_bar
import gpu_common as gc
import paper_2605_30574_amd as sp
import workloads
from oracle import decoder as ref
from paper_2605_30574_amd import decode
from workloads.model import make_weights

pytestmark = pytest.mark.gpu

LOGIT_REL = 0.008   # the decode loop's bar (test_gpu_decode.py): the attention's bar through the layers
# one more rounding of the attention's result to bf16 (2^-8 of it, as its mean error is held to 1e-3 there): added to the bar
TREE_REL = LOGIT_REL + 2.0 ** -8


def setup(name, kv="bf16", dtype=torch.float32):
    w = decode_bar.case(name)
    m = decode_bar.MODEL
    lw = workloads.cell_lw(w)
    wt = make_weights(w, m, dtype=dtype)
    on = lambda t: t.cuda()  # noqa: E731
    gpu_wt = {"embed": on(wt["embed"]), "lm_head": on(wt["lm_head"]), "norm_f": on(wt["norm_f"]),
              "layers": [{k: on(v) for k, v in L.items()} for L in wt["layers"]]}
    caches = [gc.gpu_layer(w, l, n_cells=lw.shape[0]) for l in range(w.n_layers)]
    prompts = [{k: v for k, v in gc.host(c).items() if k in ("clean_k", "clean_v", "donor_k", "donor_v")} for c in caches]
    if kv == "e4m3":
        for c in caches:
            for x in ("gen_k", "gen_v"):
                c[x + "_exp"] = torch.full(c[x].shape[:3], 127, dtype=torch.uint8, device="cuda")
                c[x] = torch.zeros(c[x].shape, dtype=torch.uint8, device="cuda")
    return w, m, lw, wt, decode.SweepDecoder(w, m, gpu_wt, caches, lw), prompts, caches


def chain(C, T):
    return np.tile(np.arange(-1, T - 1), (C, 1))


@pytest.mark.parametrize("name", decode_bar.CASES)
def test_chain_matches_the_oracle(name):
    """T tokens in one pass: the logits of T passes."""
    w, m, lw, wt, gpu, prompts, _ = setup(name)
    cpu = ref.ReferenceDecoder(w, m, decode_bar.f64_weights(wt), prompts, lw)
    C, T = lw.shape[0], min(5, w.n_steps // 2)
    rng = np.random.default_rng(3)
    tokens = rng.integers(0, m.vocab, (C, 2 * T))
    steps = np.zeros(C, np.int32)
    tree = gpu.make_tree(chain(C, T))
    for part in range(2):
        gc.announce(f"tree pass {name} part {part}")
        tok = torch.from_numpy(tokens[:, part * T:(part + 1) * T]).cuda()
        got = gpu.tree_logits(tok, tree, steps).float().cpu().numpy().reshape(C, T, -1)
        for t in range(T):
            want = cpu.forward(tokens[:, part * T + t], steps + t)
            err = np.abs(got[:, t] - want).max() / max(1.0, np.abs(want).max())
            assert err <= TREE_REL, f"{name} node {t}: logits off by {err:.2e}"
        steps = steps + T


def test_branches_are_chains_of_their_own():
    """Every node of a tree scores what it scores at the end of its path alone."""
    w, m, lw, _, gpu, _, caches = setup(decode_bar.CASES[0])
    C = lw.shape[0]
    parents = np.tile([-1, 0, 0, 1, 2, -1, 5], (C, 1))
    parents[1, 4:] = -2
    depth, words = sp.tree_layout(parents)
    T = parents.shape[1]
    rng = np.random.default_rng(5)
    tokens = torch.from_numpy(rng.integers(0, m.vocab, (C, T))).cuda()
    targets = torch.from_numpy(rng.integers(0, m.vocab, (C, T))).cuda()
    steps = np.full(C, 2, np.int32)
    steps[2] = -1
    first = gpu.make_tree(chain(C, 2))
    gpu.tree_logits(tokens[:, :2].contiguous(), first, np.zeros(C, np.int32))   # two rows behind the prompt
    tree = gpu.make_tree(parents)
    got = gpu.score_tree(tokens, tree, steps, targets, top=3)
    for t in range(T):
        path = [u for u in range(T) if (int(words[0, t]) >> u) & 1]
        alone = gpu.make_tree(chain(C, len(path)))
        want = gpu.score_tree(tokens[:, path].contiguous(), alone, steps, targets[:, path].contiguous(), top=3)
        on = torch.from_numpy((depth[:, t] >= 0) & (steps >= 0)).cuda()
        size = want.lse.abs().max()
        for f in ("lse", "entropy", "logp"):
            a, b = getattr(got, f)[on, t], getattr(want, f)[on, -1]
            assert ((a - b).abs() <= 4 * TREE_REL * size).all(), (f, t)
    assert got.top.shape == (C, T, 3) and got.rank.shape == (C, T)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_kept_nodes_are_a_plain_decode(kv):
    """Draft, accept, keep: the rows that stay are those of a chain of the accepted tokens, bit for bit at layer 0, and the
    pass behind them scores as behind that chain."""
    w, m, lw, _, gpu, _, caches = setup(decode_bar.CASES[0], kv, torch.bfloat16)
    *_, plain, _, plain_caches = setup(decode_bar.CASES[0], kv, torch.bfloat16)
    C = lw.shape[0]
    steps = np.zeros(C, np.int32)
    rng = np.random.default_rng(9)
    parents = np.tile([-1, -1, 0, 1, 1, 4], (C, 1))
    tokens = rng.integers(0, m.vocab, (C, 6))
    tree = gpu.make_tree(parents)
    tok = torch.from_numpy(tokens).cuda()
    gpu.score_tree(tok, tree, steps, tok)
    # the accepted path is 1, 4, 5 in even cells and 0 in odd ones
    best = np.full((C, 6), -1)
    best[::2, 1], best[::2, 4] = tokens[::2, 4], tokens[::2, 5]
    first = np.where(np.arange(C) % 2 == 0, tokens[:, 1], tokens[:, 0])
    tokens[::2, 0] = tokens[::2, 1] + 1   # (so that only node 1 is the root's choice; its scores are not looked at)
    keep, number = decode.accept(parents, tokens, first, best)
    assert keep[0].tolist() == [1, 4, 5, -1, -1, -1] and number[0] == 3 and number[1] == 1 and keep[1, 0] == 0
    gpu.keep_nodes(tree, steps, torch.from_numpy(keep).cuda())
    line = np.zeros((C, 3), np.int64)
    for c in range(C):
        line[c, :number[c]] = tokens[c, keep[c, :number[c]]]
    alone = plain.make_tree(np.where(np.arange(3) < number[:, None], chain(C, 3), -2))
    plain.tree_logits(torch.from_numpy(line).cuda(), alone, steps)
    torch.cuda.synchronize()
    for l in range(w.n_layers):
        for x in ("gen_k", "gen_v"):
            for c in range(C):
                a, b = caches[l][x][c, :, :number[c]], plain_caches[l][x][c, :, :number[c]]
                if l == 0:
                    assert torch.equal(a, b), (l, x, c)
    after = steps + number.astype(np.int32)
    more = torch.from_numpy(rng.integers(0, m.vocab, (C, 2))).cuda()
    two = gpu.make_tree(chain(C, 2)), plain.make_tree(chain(C, 2))
    a = gpu.tree_logits(more, two[0], after).float()
    b = plain.tree_logits(more, two[1], after).float()
    assert (a - b).abs().max() <= TREE_REL * max(1.0, float(b.abs().max()))
    if kv == "bf16":   # and the plain decode loop goes on from there
        c = gpu.forward(more[:, 0], after)
        assert (c - a.view(C, 2, -1)[:, 0]).abs().max() <= TREE_REL * max(1.0, float(c.abs().max()))


def test_scores_are_those_of_the_logits():
    w, m, lw, _, gpu, _, _ = setup(decode_bar.CASES[0], dtype=torch.bfloat16)
    C = lw.shape[0]
    tree = gpu.make_tree(chain(C, 4))
    tok = torch.randint(0, m.vocab, (C, 4), generator=torch.Generator().manual_seed(1)).cuda()
    steps = np.arange(C).astype(np.int32) % 3
    got = gpu.score_tree(tok, tree, steps, tok, top=5, scale=0.5)
    logits = gpu.tree_logits(tok, tree, steps).double()
    logp = torch.log_softmax(logits * 0.5, -1).view(C, 4, -1)
    assert (got.logp.double() - logp.gather(2, tok[..., None])[..., 0]).abs().max() < 1e-5
    assert torch.equal(got.top[..., 0], logits.argmax(-1).view(C, 4))


def test_refusals():
    w, m, lw, _, gpu, _, caches = setup(decode_bar.CASES[0])
    C = lw.shape[0]
    with pytest.raises(ValueError):
        gpu.make_tree(chain(C + 1, 2))
    with pytest.raises(ValueError):
        gpu.make_tree([[0] * 2] * C)
    tree = gpu.make_tree(chain(C, 2))
    with pytest.raises(ValueError):
        gpu.tree_logits(torch.zeros((C, 3), dtype=torch.int64, device="cuda"), tree, np.zeros(C, np.int32))
    with pytest.raises(sp.SpliceError):   # no room for the tree's rows
        gpu.tree_logits(torch.zeros((C, 2), dtype=torch.int64, device="cuda"), tree, np.full(C, w.n_steps - 1, np.int32))
    caches[0]["gen_k"] = caches[0]["gen_k"].float()
    with pytest.raises(ValueError):
        gpu.make_tree(chain(C, 2))


def test_targets_and_nodes_of_another_shape():
    w, m, lw, _, gpu, _, _ = setup(decode_bar.CASES[0])
    C, T = lw.shape[0], lw.shape[0] + 1
    steps = np.zeros(C, np.int32)
    tree = gpu.make_tree(chain(C, T))
    tokens = torch.zeros((C, T), dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        gpu.score_tree(tokens, tree, steps, tokens.t().contiguous())
    with pytest.raises(ValueError):
        gpu.keep_nodes(tree, steps, torch.zeros((T, C), dtype=torch.int32, device="cuda"))
