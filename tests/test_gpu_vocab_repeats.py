"""The losses over a vocabulary give the same bits whatever runs beside them, whatever the workspace held and however the vocabulary
is cut into pieces, in every kernel that the sizes choose between (test_kernels_of_the_sizes says which these reach)."""
import pytest
import torch

import paper_2006_16668_amd as moe
from test_gpu_vocab_loss import DEV, call, make
from test_vocab_rules import dw_on_tiles, dw_splits, dx_plan, logits_on_tiles

# S, M, V, K, dtype, share without a target
EDGE = [(40, 64, 700, 0, "bf16", 0.2), (40, 64, 700, 3, "f32", 0.2), (900, 136, 2500, 8, "bf16", 0.2), (1500, 260, 3001, 0, "f32", 0.2)]
TILES = [(1024, 1024, 32000, 0, "bf16", 0.9), (2100, 768, 17000, 32, "bf16", 0.2), (12001, 72, 1030, 0, "bf16", 0.4),
         (6011, 520, 1111, 40, "bf16", 0.4), (9001, 72, 26001, 0, "bf16", 0.3)]


def test_kernels_of_the_sizes():
    seen = set()
    for S, M, V, K, dtype, empty in EDGE + TILES:
        if dtype == "bf16":
            saved = max(0.0, 2 * S * K * M / 6e6 - 16) if 2 * S * K * M > 1e8 else 0.0
            p = dx_plan(S, V, M)
            seen |= {("z", logits_on_tiles(S, V, M, True, saved)), ("sorted", saved > 0 and logits_on_tiles(S, V, M, True, saved)),
                     ("dz", logits_on_tiles(S, V, M, False)), ("dx", p.tiles), ("dx ranges", p.splits > 1), ("dw", dw_on_tiles(S, V, M)),
                     ("dw ranges", dw_splits(S, V, M) > 1)}
    assert seen == {(k, b) for k in ("z", "sorted", "dz", "dx", "dx ranges", "dw", "dw ranges") for b in (True, False)}


@pytest.mark.gpu
@pytest.mark.parametrize("S,M,V,K,dtype,empty", EDGE + TILES)
def test_same_bits_whatever_the_workspace_held(S, M, V, K, dtype, empty):
    d = make(1, S, M, V, dtype, empty, K)
    a, *others = (call(1, S, M, V, dtype, d, K, 2.0, ws_fill=f) for f in (0x00, 0xff, 0x3f))
    for b in others:
        for k in a:
            assert torch.equal(a[k], b[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("S,M,V,K,dtype,empty", EDGE + TILES)
def test_pieces_change_no_loss(S, M, V, K, dtype, empty):
    """Nor does a vocabulary in pieces, each of which may take another kernel than the whole, make gradients that change."""
    d = make(1, S, M, V, dtype, empty, K)
    whole = call(1, S, M, V, dtype, d, K, 2.0, backward=False)
    a, b = (call(1, S, M, V, dtype, d, K, 2.0, piece=max(256, V // 3), ws_fill=f) for f in (0x00, 0xff))
    for k in a:
        assert torch.equal(a[k], b[k]), k
    for k in whole:
        assert torch.equal(a[k], whole[k]), k


class _Stream:
    """Both passes of one call on a stream of their own, in buffers and workspaces of their own, all there before the first is enqueued."""

    def __init__(self, S, M, V, K, dtype, empty, seed):
        self.d = d = make(1, S, M, V, dtype, empty, K, seed=seed)
        self.want = call(1, S, M, V, dtype, d, K, 2.0)
        self.sh, self.dims, self.K = moe.MoEShape(1, S, M, M, 2, 1, dtype), moe.VocabDims(V, K=K, temperature=2.0), K
        u8 = lambda n: torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
        self.ws = u8(moe.moe_vocab_workspace_bytes(self.sh, self.dims))
        self.bws = u8(moe.moe_vocab_backward_workspace_bytes(self.sh, self.dims))
        nan = lambda *s: torch.full((1, S, *s), float("nan"), device=DEV)
        self.x = d["x"].view(1, S, M)
        self.target, self.idx, self.logit = (d[k].view(1, S, *d[k].shape[1:]) if k in d else None for k in ("target", "idx", "logit"))
        self.dloss = d["dloss"].view(1, S)
        self.out = {"loss": nan(), "lse": nan(), "dx": torch.full_like(self.x, float("nan")), "dw": torch.full_like(d["w"], float("nan"))}
        if K:
            self.out["entry_logit"] = nan(K)
        self.stream = torch.cuda.Stream()

    def enqueue(self):
        o, w = self.out, self.d["w"]
        with torch.cuda.stream(self.stream):
            for t in o.values():
                t.fill_(float("nan"))
            if self.K:
                moe.moe_vocab_distill(self.sh, self.dims, self.x, w, self.idx, self.logit, o["loss"], o["lse"], o["entry_logit"], self.ws)
                moe.moe_vocab_distill_backward(self.sh, self.dims, self.x, w, self.idx, self.logit, o["entry_logit"], o["lse"],
                                               self.dloss, o["dx"], o["dw"], self.bws)
            else:
                moe.moe_vocab_loss(self.sh, self.dims, self.x, w, self.target, o["loss"], o["lse"], self.ws)
                moe.moe_vocab_loss_backward(self.sh, self.dims, self.x, w, self.target, o["loss"], o["lse"], self.dloss, o["dx"],
                                            o["dw"], self.bws)

    def check(self, what):
        for k, t in self.out.items():
            assert torch.equal(t.view(self.want[k].shape), self.want[k]), (what, k)


@pytest.mark.gpu
@pytest.mark.parametrize("one,other", [(EDGE[0], EDGE[1]), (EDGE[2], EDGE[3]), (TILES[0], EDGE[2]), (TILES[1], TILES[0]), (TILES[2], TILES[3])])
def test_streams_that_run_at_once(one, other):
    """Several rounds of both passes on two streams with nothing between them that waits, all enqueued before the first may start (else
    small calls are done before the host has made the next): kernels of one run beside kernels of the other.  Other inputs on each, so
    that a result in the wrong place shows."""
    moe.moe_prepare()
    jobs = [_Stream(*one, seed=3), _Stream(*other, seed=4)]
    torch.cuda.synchronize()
    start = torch.cuda.Event()
    torch.cuda._sleep(60_000_000)                                # (some 30 ms of the default stream)
    start.record()
    for j in jobs:
        j.stream.wait_event(start)
    for i in range(8):
        for j in jobs if i % 2 == 0 else jobs[::-1]:
            j.enqueue()
    torch.cuda.synchronize()
    for i, j in enumerate(jobs):
        j.check(i)
