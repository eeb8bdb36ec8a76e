"""SweepDecoder's tree passes: what a branch sees, and weights of every type that the plain decode loop takes."""
import numpy as np
import pytest
import torch

import decode_bar
import gpu_common as gc
import paper_2605_30574_amd as sp
import tree_reference
import workloads
from oracle import decoder as ref
from paper_2605_30574_amd import decode
from test_gpu_tree_pass import TREE_REL, chain
from workloads.model import make_weights

pytestmark = pytest.mark.gpu

MODEL = decode_bar.MODEL


def short_prompt():
    """A prompt of 8 slots, beside which a few nodes weigh much."""
    return decode_bar.case("blank-sink").with_(prompt_len=8, span=(2, 6))


def setup(w, dtype=torch.float32):
    lw = workloads.cell_lw(w)
    wt = make_weights(w, MODEL, dtype=dtype)
    on = lambda t: t.cuda()  # noqa: E731
    gpu_wt = {"embed": on(wt["embed"]), "lm_head": on(wt["lm_head"]), "norm_f": on(wt["norm_f"]),
              "layers": [{k: on(v) for k, v in L.items()} for L in wt["layers"]]}
    caches = [gc.gpu_layer(w, l, n_cells=lw.shape[0]) for l in range(w.n_layers)]
    prompts = [{k: v for k, v in gc.host(c).items() if k in ("clean_k", "clean_v", "donor_k", "donor_v")} for c in caches]
    return lw, wt, decode.SweepDecoder(w, MODEL, gpu_wt, caches, lw), prompts, caches


def test_branches_see_their_own_path():
    """The logits of every node are the float64 decoder's behind the node's path; behind a path with another parent that
    decoder's own are further off than four times the bar, so that a wrong branch fails here."""
    w = short_prompt()
    lw, wt, gpu, prompts, _ = setup(w)
    C, T = lw.shape[0], 7
    parents = np.tile([-1, 0, 0, 1, 2, -1, 5], (C, 1))
    depth, words = sp.tree_layout(parents)
    rng = np.random.default_rng(5)
    tokens, before = rng.integers(0, MODEL.vocab, (C, T)), rng.integers(0, MODEL.vocab, (C, 2))
    weights = decode_bar.f64_weights(wt)

    def along(path):
        cpu, steps = ref.ReferenceDecoder(w, MODEL, weights, prompts, lw), np.zeros(C, np.int32)
        for t in (*before.T, *tokens[:, path].T):
            logits = cpu.forward(t, steps)
            steps = steps + 1
        return logits

    gpu.tree_logits(torch.from_numpy(before).cuda(), gpu.make_tree(chain(C, 2)), np.zeros(C, np.int32))
    gc.announce("branches of a tree")
    steps = np.full(C, 2, np.int32)
    got = gpu.tree_logits(torch.from_numpy(tokens).cuda(), gpu.make_tree(parents), steps).double().cpu().numpy().reshape(C, T, -1)
    for t in range(T):
        path = [u for u in range(T) if (int(words[0, t]) >> u) & 1]
        want = along(path)
        size = max(1.0, np.abs(want).max())
        assert np.abs(got[:, t] - want).max() <= TREE_REL * size, f"node {t}"
        for i in range(len(path) - 1):
            for other in set(range(T)) - set(path):
                wrong = path[:i] + [other] + path[i + 1:]
                assert np.abs(along(wrong) - want).max() > 4 * TREE_REL * size, (t, wrong)


def test_ranks_and_alternatives_of_every_node():
    """score_tree's fields are those of tree_logits' rows, in float64."""
    w = short_prompt()
    lw, _, gpu, _, _ = setup(w)
    C, T, k = lw.shape[0], 7, 4
    parents = np.tile([-1, 0, 0, 1, 2, -1, 5], (C, 1))
    parents[1, 5:] = -2
    rng = np.random.default_rng(6)
    tokens, targets = (torch.from_numpy(rng.integers(0, MODEL.vocab, (C, T))).cuda() for _ in range(2))
    steps = np.arange(C).astype(np.int32)
    tree = gpu.make_tree(parents)
    got = gpu.score_tree(tokens, tree, steps, targets, top=k)
    x = gpu.tree_logits(tokens, tree, steps).double().cpu().numpy()
    logp, lse, entropy, rank, top, top_logp = tree_reference.scores(x, targets.reshape(-1).cpu().numpy(), k)
    on = (parents >= -1).reshape(-1)
    assert np.array_equal(got.rank.reshape(-1).cpu().numpy()[on], rank[on])
    assert np.array_equal(got.top.reshape(-1, k).cpu().numpy()[on], top[on])
    for name, want in (("logp", logp), ("lse", lse), ("entropy", entropy), ("top_logp", top_logp)):
        assert np.abs(getattr(got, name).double().cpu().numpy().reshape(want.shape) - want)[on].max() < 1e-4, name


@pytest.mark.parametrize("dtype,cast", [(torch.float16, False), (torch.float64, False), (torch.bfloat16, True), (torch.float32, True)])
def test_weights_of_other_types_are_scored(dtype, cast):
    """What forward takes, score_tree takes: weights in other types than bfloat16 and float32, products under autocast."""
    w = decode_bar.case("blank-sink")
    lw, _, gpu, _, _ = setup(w, dtype)
    *_, plain, _, _ = setup(w, dtype)
    C, T = lw.shape[0], 4
    tokens = torch.randint(0, MODEL.vocab, (C, T), generator=torch.Generator().manual_seed(1)).cuda()
    steps, tree = np.zeros(C, np.int32), gpu.make_tree(chain(C, T))
    gc.announce(f"tree scores with weights of {dtype}, autocast {cast}")
    with torch.autocast("cuda", torch.float16, enabled=cast):
        got = gpu.score_tree(tokens, tree, steps, tokens, top=3)
        logits = gpu.tree_logits(tokens, tree, steps)
        want = [plain.forward(tokens[:, t], steps + t) for t in range(T)]
    logp = torch.log_softmax(logits.double(), -1).view(C, T, -1)
    assert (got.logp.double() - logp.gather(2, tokens[..., None])[..., 0]).abs().max() < 1e-5
    assert torch.equal(got.top[..., 0], logits.argmax(-1).view(C, T))
    for t in range(T):   # each side is off by its own bar from the float64 decoder
        err = (logits.view(C, T, -1)[:, t].double() - want[t].double()).abs().max()
        assert err <= 2 * TREE_REL * max(1.0, float(want[t].abs().max())), t


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("own_positions", [False, True])
def test_keys_of_the_first_layer_are_rounded_once(dtype, own_positions):
    """Where the products have more bits than bfloat16, keys are rotated before they are rounded, as a decode step's are."""
    w = decode_bar.case("blank-sink")
    lw, _, gpu, _, caches = setup(w, dtype)
    C, T, D, Hkv = lw.shape[0], 6, w.head_dim, w.n_kv_heads
    ahead = 1000 if own_positions else 0
    if own_positions:
        plain = gpu.positions
        gpu.positions = lambda steps: plain(steps) + ahead
    rng = np.random.default_rng(8)
    parents = np.array([[-1] + [int(rng.integers(0, t)) for t in range(1, T)] for _ in range(C)])
    tokens = torch.from_numpy(rng.integers(0, MODEL.vocab, (C, T))).cuda()
    steps = rng.integers(0, w.n_steps - T + 1, C).astype(np.int32)
    gc.announce(f"keys of layer 0, {dtype}, own positions {own_positions}")
    gpu.tree_logits(tokens, gpu.make_tree(parents), steps)
    p = gpu.wt["layers"][0]
    h = decode.rms_norm(gpu.wt["embed"][tokens.reshape(-1)].float(), p["norm_1"], MODEL.rms_eps).to(dtype)
    k = (h @ p["w_k"]).double().cpu().numpy().reshape(C, T, Hkv, D)   # the product whose rotation the rows hold
    depth, _ = sp.tree_layout(parents)
    pos = np.broadcast_to((w.prompt_len + ahead + steps[:, None] + depth)[..., None], k.shape[:3])
    want = tree_reference.rotated(k, pos, MODEL.rope_theta ** (-np.arange(0, D, 2) / D), "half", D, 1.0)
    # half a step of the result; of the pair's values, the angle's half step in float32 and the rotation's roundings
    pair = np.abs(k) + np.abs(np.roll(k, D // 2, -1))
    tol = 2.0 ** -8 * np.abs(want) + (pos[..., None] * 2.0 ** -24 + 2.0 ** -20) * pair
    got = caches[0]["gen_k"].double().cpu().numpy()
    for c in range(C):
        off = np.abs(got[c, :, steps[c]:steps[c] + T].transpose(1, 0, 2) - want[c]) - tol[c]
        assert (off <= 0).all(), f"cell {c}: off by {off.max():.3e} more than it may be"


def test_captured_pass_with_float32_weights():
    """A captured pass of the written-out form, replayed on other tokens between eager ones: the eager bits."""
    w = decode_bar.case("blank-sink")
    lw, _, gpu, _, caches = setup(w)
    C, T = lw.shape[0], 5
    tree, steps = gpu.make_tree(chain(C, T)), np.arange(C).astype(np.int32)
    tokens = torch.zeros((C, T), dtype=torch.int64, device="cuda")
    gpu.tree_logits(tokens, tree, steps)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = gpu.tree_logits(tokens, tree, steps)
    for n in range(3):
        gc.announce(f"captured float32 tree pass, replay {n}")
        tokens.copy_(torch.randint(0, MODEL.vocab, (C, T), generator=torch.Generator().manual_seed(n)))
        graph.replay()
        torch.cuda.synchronize()
        got, rows = logits.clone(), [c["gen_k"].clone() for c in caches]
        assert torch.equal(got, gpu.tree_logits(tokens, tree, steps))
        torch.cuda.synchronize()
        assert all(torch.equal(a, c["gen_k"]) for a, c in zip(rows, caches))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["stretched", "between", "by cell"])
def test_positions_of_the_decoders_own(kind, dtype):
    """A node's position is what positions() says of its step, whatever that is: the keys and logits of a chain are those of
    decode steps."""
    w = decode_bar.case("blank-sink")
    lw, _, gpu, _, caches = setup(w, dtype)
    *_, plain, _, plain_caches = setup(w, dtype)
    C, T, D = lw.shape[0], 5, w.head_dim
    cell = np.arange(C)
    own = {"stretched": lambda s: w.prompt_len + 3 * np.maximum(s, 0), "between": lambda s: (w.prompt_len + np.maximum(s, 0)) / 4,
           "by cell": lambda s: w.prompt_len + cell + (1 + cell % 2) * np.maximum(s, 0)}[kind]
    for d in (gpu, plain):
        d.positions = lambda s: torch.as_tensor(own(s)).cuda()
    tokens = torch.randint(0, MODEL.vocab, (C, T), generator=torch.Generator().manual_seed(2)).cuda()
    steps = np.arange(C).astype(np.int32)
    gc.announce(f"positions {kind}, {dtype}")
    got = gpu.tree_logits(tokens, gpu.make_tree(chain(C, T)), steps).view(C, T, -1).double()
    for t in range(T):
        want = plain.forward(tokens[:, t], steps + t).double()
        assert (got[:, t] - want).abs().max() <= 2 * TREE_REL * max(1.0, float(want.abs().max())), t
    # two roundings to bf16 of a rotation, whose pairs keep their length, and their products' own
    a, b = (x[0]["gen_k"].double().cpu().numpy() for x in (caches, plain_caches))
    length = np.hypot(b, np.roll(b, D // 2, -1))
    assert (length > 0).any() and (np.abs(a - b) <= 2.0 ** -6 * length).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_pass_with_positions_on_the_device(dtype):
    """positions() that makes no copy from the host is asked within a captured pass; cells that are finished and padding too."""
    w = decode_bar.case("blank-sink")
    lw, _, gpu, _, _ = setup(w, dtype)
    C = lw.shape[0]
    table = (torch.arange(w.n_steps * C, device="cuda").view(w.n_steps, C) * 5) % 97   # [step][cell]
    steps = np.full(C, 3, np.int32)
    steps[1] = -1
    gpu.positions = lambda s: table[int(s.max())]
    parents = np.tile([-1, 0, 0, 2, -1], (C, 1))
    parents[2, 3:] = -2
    tree, tokens = gpu.make_tree(parents), torch.zeros((C, 5), dtype=torch.int64, device="cuda")
    gpu.tree_logits(tokens, tree, steps)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = gpu.tree_logits(tokens, tree, steps)
    on = torch.from_numpy(((parents >= -1) & (steps >= 0)[:, None]).reshape(-1)).cuda()
    for n in range(3):
        gc.announce(f"captured tree pass, positions on the device, {dtype}, replay {n}")
        tokens.copy_(torch.randint(0, MODEL.vocab, tokens.shape, generator=torch.Generator().manual_seed(n)))
        table.add_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = logits.clone()
        assert torch.equal(got[on], gpu.tree_logits(tokens, tree, steps)[on])
        torch.cuda.synchronize()
