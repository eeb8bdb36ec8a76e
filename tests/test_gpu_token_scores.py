"""splice_token_scores against the definition in float64."""
import numpy as np
import pytest
import torch

from tree_common import announce, f64, ref, sp

pytestmark = pytest.mark.gpu


def check(logits, tokens, k, scale=1.0, got=None):
    got = got or sp.token_scores(logits, tokens, k, scale)
    torch.cuda.synchronize()
    raw = f64(logits)
    vocab = raw.shape[1]
    logp, lse, entropy, rank, top, top_logp = ref.scores(raw * scale, tokens.cpu().numpy(), k)
    fine = np.isfinite(raw * scale)
    size = np.abs(np.where(fine, raw * scale, 0)).max(-1)
    # x log2(e) scale in one rounding each (3 * 2^-24 of |x|), v_exp_f32 and v_log_f32 (2^-22), sums of vocab weights in
    # a tree under chains of vocab / 256 terms
    tol = 2.0 ** -24 * (8 * size + vocab / 256 + 64)
    def same(a, b, t):
        a = f64(a)
        ok = (np.isnan(a) & np.isnan(b)) | (a == b) | (np.abs(a - b) <= t)
        assert ok.all(), (a[~ok][:4], b[~ok][:4])
    same(got.lse, lse, tol)
    same(got.logp, logp, 2 * tol)
    # entropy: sum p (lse - x), the weights' errors times the distances
    same(got.entropy, entropy, 2 * tol * (1 + np.log(vocab) + np.abs(np.nan_to_num(entropy))))
    assert np.array_equal(got.rank.cpu().numpy(), rank)
    if k:
        assert np.array_equal(got.top.cpu().numpy(), top)
        same(got.top_logp, top_logp, 2 * tol[:, None])
    else:
        assert got.top is None and got.top_logp is None


def draw(seed, rows, vocab, dtype, spread=2.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocab + pad, generator=g) * spread).to(dtype).cuda()
    return x[:, pad // 2:pad // 2 + vocab], torch.randint(0, vocab, (rows,), generator=g).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (5, 7, 0), (4, 63, 63), (2, 64, 64), (3, 65, 5), (1, 1000, 64),
                                          (2, 8192, 20), (7, 8193, 1), (3, 33333, 64), (40, 4097, 3)])
def test_sizes(rows, vocab, k, dtype):
    announce(f"scores {rows} {vocab} {k} {dtype}")
    check(*draw(vocab, rows, vocab, dtype), k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 2, 3, 5, 8, 15])
def test_rows_at_any_offset(pad, dtype):
    check(*draw(pad, 6, 1001, dtype, pad=pad), 4, 0.7)


def test_ties_go_to_the_lower_index():
    x = torch.zeros(4, 5000, device="cuda")
    x[1] = -3.0
    x[1, 17::100] = 2.5
    x[2] = torch.randint(0, 3, (5000,), generator=torch.Generator().manual_seed(3)).float()
    x[3, ::2] = -0.0
    check(x, torch.tensor([4999, 117, 2500, 1], device="cuda"), 64)
    check(x.to(torch.bfloat16), torch.tensor([0, 18, 4999, 0], device="cuda"), 64)


def test_masked_infinite_and_nan():
    x, t = draw(5, 12, 3000, torch.float32)
    x = x.contiguous()
    x[0] = -np.inf
    x[1, 5:] = -np.inf
    x[2, 1:] = -np.inf
    x[3, 100] = np.inf
    x[4, 7] = np.nan
    x[5, 2999] = np.nan
    x[5, 3] = np.nan
    x[6] = torch.finfo(torch.float32).min
    x[7, :2000] = torch.finfo(torch.float32).min
    x[8] = np.nan
    x[9, ::3] = -np.inf
    t[1], t[2], t[4], t[5], t[9] = 200, 0, 7, 2999, 0
    t[10], t[11] = -1, 3000   # no tokens
    check(x, t, 8)
    check(x.to(torch.bfloat16), t, 8)


def test_peaked_and_flat_entropy():
    x = torch.zeros(3, 4000, device="cuda")
    x[0, 9] = 60.0
    x[1, 9] = 15.0
    check(x, torch.tensor([9, 8, 7], device="cuda"), 2)


def test_scale_and_large_logits():
    x, t = draw(6, 4, 999, torch.float32, spread=300.0)
    for scale in (0.01, 1.0, 7.5):
        check(x, t, 10, scale)


def test_token_chunk_borders():
    """The given token at either end of a 16-byte chunk and of a part, among equals."""
    x = torch.zeros(40, 20000, device="cuda")
    t = torch.tensor([0, 1, 3, 4, 5, 1023, 1024, 4095, 4096, 4097, 8191, 8192, 9999, 10000, 19996, 19999, 12, 15, 16, 17] * 2, device="cuda")
    x[20:, ::2] = 1.0
    check(x, t, 1)
    check(x.to(torch.bfloat16), t, 1)


def test_replayed_graph_and_same_bits():
    x, t = draw(8, 3, 50000, torch.bfloat16)
    x, ws = x.contiguous(), torch.empty(sp.splice_token_scores_workspace_bytes(3, 50000, 5), dtype=torch.uint8, device="cuda")
    o = [torch.empty(3, device="cuda") for _ in range(3)] + [torch.empty(3, dtype=torch.int64, device="cuda"),
                                                           torch.empty(3, 5, dtype=torch.int64, device="cuda"), torch.empty(3, 5, device="cuda")]
    run = lambda: sp.splice_token_scores(x, t, *o, ws)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for n in range(3):
        x.copy_(draw(20 + n, 3, 50000, torch.bfloat16)[0])
        graph.replay()
        torch.cuda.synchronize()
        eager = sp.token_scores(x, t, 5)
        torch.cuda.synchronize()
        for a, b in zip(o, eager):
            assert torch.equal(a, b)
        check(x, t, 5, got=sp.TokenScores(*o))


@pytest.mark.parametrize("k", [1, 7, 20, 64])
@pytest.mark.parametrize("kind", ["rising", "falling", "constant", "steps", "late"])
@pytest.mark.parametrize("rows", [1, 3, 1100])
def test_candidates_in_any_order(rows, kind, k):
    """Rows whose candidates fill a wave's list again and again, or come all at the end; as one part and as several."""
    vocab = 33000 if rows < 100 else 9000
    i = torch.arange(vocab, dtype=torch.float32)
    x = {"rising": i / vocab, "falling": -i / vocab, "constant": i * 0, "steps": torch.floor(i / 97),
         "late": torch.where(i < vocab - 300, i * 0 - 5, torch.sin(i))}[kind]
    x = x.repeat(rows, 1).cuda()
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(k)).cuda()
    got = sp.token_scores(x, t, k)
    check(x[:1], t[:1], k, got=sp.TokenScores(*(f[:1] for f in got)))
    torch.cuda.synchronize()
    for f in (got.lse, got.entropy, got.top, got.top_logp):   # the same row: the same bits
        assert torch.equal(f, f[:1].expand_as(f))


def exact_in_distances(logits, tokens, k, scale=1.0):
    """Like check, with tolerances that do not grow with the logits: log s is off by the sums' 2^-24 vocab / 256, 64 for v_exp_f32,
    v_log_f32 and the joins, 96 for a reference of up to 256 rounded once (2^-17 ln 2 = 89 * 2^-24), and three roundings of each
    distance, which the weights sum to less than ln vocab; a distance (x - m) scale by four roundings, lse by two."""
    got = sp.token_scores(logits, tokens, k, scale)
    torch.cuda.synchronize()
    raw = f64(logits)
    most, t = raw.max(-1), tokens.cpu().numpy()
    # (in float64 too a log-sum of some 1e20 would lose the logarithm that log probabilities are made of, and distances from it the
    # order of what is near 0)
    logp, lse, entropy, _, _, top_logp = ref.scores((raw - most[:, None]) * scale, t, k)
    _, _, _, rank, top, _ = ref.scores(raw, t, k)
    lse = most * scale + lse
    vocab = raw.shape[1]
    tol = 2.0 ** -24 * (vocab / 256 + 64 + 96 + 3 * np.log(vocab))

    def near(name, want, bound):
        a = f64(getattr(got, name))
        assert np.isfinite(a).all(), (name, a)
        assert (np.abs(a - want) <= bound).all(), (name, a, want)
    near("lse", lse, tol + 2.0 ** -23 * np.abs(lse))
    near("logp", logp, tol + 2.0 ** -22 * np.abs(logp))
    near("entropy", entropy, 2 * tol * (1 + np.log(vocab) + entropy))
    assert np.array_equal(got.rank.cpu().numpy(), rank) and np.array_equal(got.top.cpu().numpy(), top)
    near("top_logp", top_logp, tol + 2.0 ** -22 * np.abs(top_logp))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,pad", [(1001, 0), (1001, 3), (20003, 5)])
def test_logits_near_the_largest_float(vocab, pad, dtype):
    """A forced token: the largest number of the type at a row's first and last values, within it, twice, and beside the lowest."""
    announce(f"largest logits {vocab} {pad} {dtype}")
    big = torch.finfo(dtype).max
    x, t = draw(vocab + pad, 12, vocab, dtype, pad=pad)
    at = [0, 1, 2, 7, vocab // 2, vocab // 2 + 5, vocab - 1, vocab - 2, vocab - 6]
    for r, i in enumerate(at):
        x[r, i] = big
        t[r] = i if r % 2 == 0 else (i + 9) % vocab
    x[9, 5], x[9, vocab - 5] = big, big
    t[9] = 5
    x[10] = -big
    x[10, 11] = big
    t[10] = 11
    x[11] = big
    exact_in_distances(x, t, 1)   # (the others' log probabilities are beyond float's range where the lowest float is among them)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [300.0, -300.0, 3.0e6, 1.0e10, -1.0e10, 1.0e20, 1.0e38, -1.0e38])
def test_logits_far_from_zero(size, dtype):
    """What a row's values have in common does not reach its probabilities."""
    announce(f"logits about {size} {dtype}")
    for vocab in (1001, 20003):
        x, t = draw(int(abs(size)) % 9973, 4, vocab, torch.float32)
        x = (x + size).to(dtype)
        x[1] = size
        exact_in_distances(x, t, 3)


def test_scale_that_takes_the_largest_logit_near_the_largest_float():
    """scale * logit is a float, and not so with the factor log2(e)."""
    x = torch.full((3, 2000), -2.0e30, device="cuda")
    x[0, 7] = x[0, 1500] = 1.0e30
    x[1, ::3] = 1.0e30
    x[2] = 1.0e30
    exact_in_distances(x, torch.tensor([7, 3, 5], device="cuda"), 2, float(np.float32(3.0e8)))
