"""The decode path over an 8-bit cache (kvdtype "fp8"): dual steps, batches,
exits, chunks, drafts, the no-allocation step and graphs, against the oracle
with a cache that quantises as the operators define (tests/kv8_ref.py).

Both sides attend over the same loaded codes.  A new entry whose value differs
by a relative d between the sides (d: the tolerance of gpu_harness) falls on
the other side of a rounding border with probability at most d / 2^-4, and is
then off by a code step, at most 2^-3 of itself: sqrt(16 d) / 8 in the norm,
2^-3 of an element, and of a subnormal code one step, 2^-9 of the scale.  That
(and d) bounds the cache entries, and what a step that sees them computes."""
import numpy as np
import pytest
import torch

import synth
from oracle import KVCache
from oracle.decoder import argmax_first
from paper_2502_02040_amd import M2R2Error, Model, PagedKV, workspace_size
from tests import kv8_ref
from tests.gpu_harness import Pair, Tally, rel, shuffled_table, token_decidable, tol_of, track
from tests.test_gpu_batch import batch_step

pytestmark = pytest.mark.gpu


class Cache8(KVCache):
    """The oracle's cache of one sequence, in 8 bits."""

    def __init__(self, cfg, max_len, block):
        super().__init__(cfg, max_len)
        self.bs, n = block, -(-max_len // block)
        self.table = np.arange(n)
        self.layers = [kv8_ref.Cache([np.zeros((n, cfg.n_heads, block, cfg.head_dim))] * 2,
                                     [np.ones((n, cfg.n_heads))] * 2) for _ in range(cfg.n_layers)]

    def write(self, l, pos, k, v):
        p0, many = (pos.start, True) if isinstance(pos, slice) else (int(pos), False)
        for which, x, out in ((0, k, self.K), (1, v, self.V)):
            y = (x if many else x[None]).astype(np.float32)
            self.layers[l].append(which, self.table, p0, y)
            b0 = p0 // self.bs * self.bs
            b1 = min(len(out[l]), -(-(p0 + len(y)) // self.bs) * self.bs)
            out[l][b0:b1] = self.layers[l].values(which, self.table, b1)[b0:]

    def load(self, l, K, V, start=0):
        self.write(l, slice(start, start + len(K)), K, V)


class Pair8(Pair):
    def __init__(self, cfg, weights, *, block_size=16, **kw):
        super().__init__(cfg, weights, block_size=block_size, **kw)
        self.caches = [Cache8(cfg, -(-self.max_ctx // block_size) * block_size, block_size) for _ in self.caches]
        d = tol_of(cfg)
        self.tol = d + np.sqrt(16 * d) / 8

    def check_cache(self, seq, start, end, tally, what=""):
        for l in range(self.cfg.n_layers):
            for which, got in enumerate(self.kv.read(seq, l, start, end)):
                c = self.caches[seq]
                ref = (c.V if which else c.K)[l][start:end]
                scale = 2.0 ** c.layers[l].exps[which][np.arange(start, end) // c.bs].astype(float)[..., None]
                most = np.abs(ref).max(axis=-1, keepdims=True)
                d = tol_of(self.cfg)
                assert np.all(np.abs(got - ref) <= d * most + 2.0 ** -3 * np.abs(ref) + 2.0 ** -9 * scale * 2), (what, l, which)
                e = rel(got, ref)
                assert e <= self.tol, f"{what} layer {l}: {e}"
                tally.worst = max(tally.worst, e)
                tally.arrays += 1


F8 = dict(kvdtype="fp8")
CONFIGS = {
    "hd64_f32": synth.CONFIGS["tiny"].replace(name="hd64_f32", **F8),
    "hd96_f32": synth.CONFIGS["small_bf16"].replace(name="hd96_f32", wdtype="f32", **F8),
    "hd128_f32": synth.CONFIGS["small_rw"].replace(name="hd128_f32", wdtype="f32", **F8),
    "hd96_bf16": synth.CONFIGS["small_bf16"].replace(name="hd96_bf16", **F8),
    "hd128_bf16": synth.CONFIGS["small_rw"].replace(name="hd128_bf16", **F8),
}


def pair_of(cfg, cap, *, n=1, block=16, seed=3):
    return Pair8(cfg, synth.make_weights(cfg), max_ctx=cap, block_size=block, max_batch=n, n_seqs=n, table_seed=seed)


@pytest.mark.parametrize("name", CONFIGS)
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 31, 127, 128, 300])
def test_one_sequence(name, ctx):
    pair, t = pair_of(CONFIGS[name], ctx + 20), Tally()
    batch_step(pair, [ctx], t)
    assert t.steps == 1


@pytest.mark.parametrize("name", ["hd64_f32", "hd96_bf16", "hd128_f32"])
@pytest.mark.parametrize("lens,block", [((0, 1, 31, 32, 33), 16), ((127, 128, 129), 48),
                                        ((255, 257, 300, 511, 640, 2, 16, 1000), 64)])
def test_batches(name, lens, block):
    pair, t = pair_of(CONFIGS[name], max(lens) + 20, n=len(lens), block=block), Tally()
    batch_step(pair, lens, t)
    assert t.steps == len(lens)


@pytest.mark.parametrize("rank,d,H,F", [(8, 544, 3, 608), (12, 544, 3, 608)])
def test_other_projections(rank, d, H, F):
    """Rows of no whole 1 KB pieces (the stream-K projections), adapter rows of no whole 16 bytes."""
    cfg = synth.CONFIGS["small_bf16"].replace(name="s8", d_model=d, n_heads=H, ffn=F, rank=rank, **F8)
    t = Tally()
    batch_step(pair_of(cfg, 256), [200], t)
    batch_step(pair_of(cfg.replace(wdtype="f32"), 256), [33], t)
    assert t.steps == 2


def test_batch_with_exits():
    """Some sequences leave at the first gate: their later layers' entries are still written, nothing else of theirs runs."""
    cfg = CONFIGS["hd64_f32"].replace(name="exit8", n_layers=4)
    lens = [40, 3, 77, 20]
    pair, t = pair_of(cfg, 100, n=4), Tally()
    n = batch_step(pair, lens, t, mode="exit", gates=[1, 2, 3], pick=lambda s: (s[1] + s[2]) / 2)
    assert n >= 1 and t.steps == 4


@pytest.mark.parametrize("name", ["hd64_f32", "hd96_bf16", "hd128_f32"])
@pytest.mark.parametrize("ctx,n", [(0, 3), (0, 16), (1, 15), (31, 7), (129, 16), (700, 5)])
def test_chunks(name, ctx, n):
    cfg = CONFIGS[name]
    pair, t = pair_of(cfg, ctx + 40), Tally()
    if ctx:
        for l, (K, V) in synth.synthetic_kv(cfg, ctx).items():
            pair.kv.load(0, l, K, V)
            pair.caches[0].load(l, K, V)
    toks = [int(x) for x in synth.prompt_ids(cfg, n, seed=9)]
    pos, targets = torch.tensor([ctx], dtype=torch.int32, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    pair.model.verify(torch.tensor(toks, dtype=torch.int32, device="cuda"), n, pos, pair.kv.desc(), targets)
    torch.cuda.synchronize()
    ref = pair.orc.slow_chunk(toks, ctx, pair.caches[0])
    for i in range(n):
        t.token(int(targets[i].item()), ref[i], pair.tol, f"row {i}")
    pair.check_cache(0, ctx, ctx + n, t)
    assert int(pos.item()) == ctx + n == int(pair.kv.seq_lens[0].item())


@pytest.mark.parametrize("ctx", [20, 61])
def test_draft_then_verify(ctx):
    """Drafts see the drafts before them in the cache; the verification overwrites their entries, in blocks whose scales
    the drafts may have raised."""
    cfg = CONFIGS["hd64_f32"].replace(name="draft8", n_layers=3)
    pair, t = pair_of(cfg, ctx + 30), Tally()
    pair.prefill([int(x) for x in synth.prompt_ids(cfg, ctx)], tally=t)
    pair.check_cache(0, 0, ctx, t)
    gamma, k, dev, c = 4, 2, pair.dev, pair.caches[0]
    last = torch.tensor([7], dtype=torch.int32, device=dev)
    pos, drafts = torch.tensor([ctx], dtype=torch.int32, device=dev), torch.zeros(gamma, dtype=torch.int32, device=dev)
    pair.model.draft(last, pos, k, gamma, pair.kv.desc(), drafts)
    torch.cuda.synchronize()
    got, tok = [int(x) for x in drafts.cpu()], 7
    for j in range(gamma):
        p = pair.orc.w["embed"][tok].copy()
        for l in range(k):
            p, (kk, vv) = pair.orc._fast_layer(l, p, ctx + j, c.K[l][:ctx + j], c.V[l][:ctx + j])
            c.write(l, ctx + j, kk, vv)
        z = pair.orc.head_logits(p)
        t.token(got[j], z, pair.tol, f"draft {j}")
        tok = got[j]
    chunk = [7] + got
    targets, n_acc = torch.zeros(16, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    pair.model.verify(torch.tensor(chunk, dtype=torch.int32, device=dev), gamma + 1, pos, pair.kv.desc(), targets, n_acc)
    torch.cuda.synchronize()
    ref = pair.orc.slow_chunk(chunk, ctx, c)
    for i in range(gamma + 1):
        t.token(int(targets[i].item()), ref[i], pair.tol, f"row {i}")
        if token_decidable(ref[i], pair.tol):
            assert int(targets[i].item()) == argmax_first(ref[i])
    pair.check_cache(0, ctx, ctx + gamma + 1, t)
    assert int(pair.kv.seq_lens[0].item()) == ctx + int(n_acc.item()) + 1


def test_steps_replayed_from_a_graph_and_without_allocation():
    """Twelve dual steps of two sequences: eager, replayed from one captured step, and through m2r2_decode_step_noalloc.  The
    statistics' atomics make passes differ in the last bits, so the states are compared, not the bytes."""
    cfg = CONFIGS["hd128_bf16"]
    w, lens, B = synth.make_weights(cfg), [30, 9], 2
    dev = torch.device("cuda")
    runs = []
    for how in ("eager", "graph", "noalloc"):
        m = track(Model(cfg, w, max_batch=B, max_chunk=16, max_ctx=64))
        kv = PagedKV(cfg, B, 64, block_table=shuffled_table(B, 64, 16, 5))
        for s, n in enumerate(lens):
            for l, (K, V) in synth.synthetic_kv(cfg, n, seq=s).items():
                kv.load(s, l, K, V)
        pos = torch.tensor(lens, dtype=torch.int32, device=dev)
        tok = torch.tensor([3, 5], dtype=torch.int32, device=dev)
        nxt = torch.zeros(B, dtype=torch.int32, device=dev)
        h = torch.zeros(B * cfg.d_model, device=dev)

        def step(stream=None):
            m.decode_step(tok, pos, kv.desc(), gates=[1, 2], mode="observe", next_token=nxt, h_out=h, advance=True,
                          noalloc=how == "noalloc", stream=stream)

        hs = []
        if how == "graph":
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(side)
        for i in range(12):
            tok.copy_(torch.tensor([3 + i, 5 + 2 * i], dtype=torch.int32))   # teacher-forced
            torch.cuda.synchronize()
            graph.replay() if how == "graph" else step()
            torch.cuda.synchronize()
            hs.append(h.cpu().numpy().copy())
        assert pos.tolist() == [n + 12 for n in lens]
        runs.append(hs)
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert rel(b, a) <= 2e-2


def test_long_context_takes_the_8_bit_path_alone():
    """A capacity above what the other caches' short-chain attention holds, on the operators: the attention of one layer's
    loaded cache equals a step's (one layer, fast row off)."""
    cfg = CONFIGS["hd128_bf16"].replace(name="long8", n_layers=1)
    pair, t = pair_of(cfg, 9000, block=64), Tally()
    batch_step(pair, [8777], t, gates=[], mode="off")
    assert t.steps == 1


def test_refusals():
    moe = synth.CONFIGS["small_moe"].replace(**F8)
    for cfg in (moe, synth.CONFIGS["tiny_flops"].replace(**F8)):
        with pytest.raises(M2R2Error) as e:
            workspace_size(cfg, 1, 16, 64)
        assert e.value.status == -7
    cfg = CONFIGS["hd64_f32"]
    m = track(Model(cfg, synth.make_weights(cfg), max_ctx=64))
    one, nxt = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for change, status in ((dict(block_size=24), -2), (dict(k_scales=None), -1), (dict(block_size=512), -2)):
        d = PagedKV(cfg, 1, 64).desc()
        for k, v in change.items():
            setattr(d, k, v)
        with pytest.raises(M2R2Error) as e:
            m.decode_step(one, one.clone(), d, next_token=nxt)
        assert e.value.status == status
