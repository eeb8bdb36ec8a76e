"""SweepDecoder's tree passes with weights of every type that the plain decode loop takes."""
import numpy as np
import pytest
import torch

import decode_bar
import gpu_common as gc
import workloads
from paper_2605_30574_amd import decode
from test_gpu_tree_pass import TREE_REL, chain
from workloads.model import make_weights

pytestmark = pytest.mark.gpu

MODEL = decode_bar.MODEL


def setup(w, dtype=torch.float32):
    lw = workloads.cell_lw(w)
    wt = make_weights(w, MODEL, dtype=dtype)
    on = lambda t: t.cuda()  # noqa: E731
    gpu_wt = {"embed": on(wt["embed"]), "lm_head": on(wt["lm_head"]), "norm_f": on(wt["norm_f"]),
              "layers": [{k: on(v) for k, v in L.items()} for L in wt["layers"]]}
    caches = [gc.gpu_layer(w, l, n_cells=lw.shape[0]) for l in range(w.n_layers)]
    prompts = [{k: v for k, v in gc.host(c).items() if k in ("clean_k", "clean_v", "donor_k", "donor_v")} for c in caches]
    return lw, wt, decode.SweepDecoder(w, MODEL, gpu_wt, caches, lw), prompts, caches


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
