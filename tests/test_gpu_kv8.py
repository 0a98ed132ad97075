"""The 8-bit cache's operators on the GPU against float64 NumPy (tests/kv8_ref.py).

Appending is compared bit for bit.  Attention's bound, per row and head, is
worst-case arithmetic (u = 2^-24, half a step of float32):
  scores   |dz| <= u (hd + 16) scale max_t sum_d |q_d k_td| + 8 u max_t |z_t|
           (products exact; a float32 sum of hd terms; scale, maximum and the exponential's argument)
  weights  each off by at most 2 |dz| + e_p relative to the sum, e_p the rounding of a probability: 2^-16 (two
           bfloat16 parts), 2^-8 (one: bfloat16 rows of many columns), 2^-23 (float32 rows)
  sums     of n positions and the joins: 2 u (n + 128)
so |out - ref| <= vmax (2 |dz| + e_p + 2 u (n + 128)) + h |ref|, h half a step of the result's type.
"""
import pathlib
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2502_02040_amd import KV8Pages, kv8_append, kv8_attention, kv8_workspace
from tests import kv8_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pool:
    """A cache of random codes (every one but NaN) and scales, with a shuffled table."""

    def __init__(self, seed, seqs, blocks, H, hd, bs, scales=(-3, 3)):
        self.rng = rng = np.random.default_rng(seed)
        n = seqs * blocks + 1
        self.codes = []
        for _ in range(2):
            c = rng.integers(0, 254, (n, H, bs, hd)).astype(np.uint8)
            self.codes.append(np.where(c >= 0x7f, c + 1, c).astype(np.uint8))
        self.scales = [2.0 ** rng.integers(scales[0] - 6, scales[1] - 6, (n, H)).astype(np.float64) for _ in range(2)]
        self.table = rng.permutation(n)[:seqs * blocks].reshape(seqs, blocks).astype(np.int32)
        self.H, self.hd, self.bs = H, hd, bs

    def upload(self):
        c = [torch.tensor(x, device="cuda").view(torch.float8_e4m3fn) for x in self.codes]
        s = [torch.tensor(x, dtype=torch.float32, device="cuda") for x in self.scales]
        self.kv = KV8Pages(c[0], c[1], s[0], s[1], i32(self.table))
        return self.kv

    def ref(self):
        return kv8_ref.Cache(self.codes, self.scales)


def rope_table(n, hd):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, hd, 2) / hd)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def same_cache(kv, ref):
    for c, e, codes, exps in ((kv.k_pages, kv.k_scales, ref.codes[0], ref.exps[0]),
                              (kv.v_pages, kv.v_scales, ref.codes[1], ref.exps[1])):
        got = kv8_ref.CODE[c.view(torch.uint8).cpu().numpy()]
        assert np.array_equal(got, kv8_ref.CODE[codes], equal_nan=True)
        assert np.array_equal(e.double().cpu().numpy(), 2.0 ** exps)


def append_both(pool, ref, dt, counts, positions, k, v, rope=None, q=None, **kw):
    start = np.concatenate([[0], np.cumsum(counts)])
    kd, vd = (torch.tensor(x).to(DT[dt]).cuda() for x in (k, v))
    qd = qo = None
    if q is not None:
        qd = torch.tensor(q).to(DT[dt]).cuda()
        qo = torch.full_like(qd, 7.0)
    kv8_append(pool.kv, kd, vd, i32(start), i32(positions), rope=None if rope is None else torch.tensor(rope).cuda(),
               q=qd, q_out=qo, **kw)
    kf, vf = kd.float().cpu().numpy(), vd.float().cpu().numpy()
    for s, p0 in enumerate(positions):
        r = slice(start[s], start[s + 1])
        if counts[s]:
            cs = None if rope is None else rope[p0:p0 + counts[s]]
            ref.append(0, pool.table[s], p0, kf[r] if rope is None else kv8_ref.rotate(kf[r], cs))
            ref.append(1, pool.table[s], p0, vf[r])
            if q is not None:
                want = qd[r].float().cpu().numpy()
                want = want if rope is None else kv8_ref.rotate(want, cs)
                assert torch.equal(qo[r].cpu(), torch.tensor(want).to(DT[dt]))
    return qo


@pytest.mark.parametrize("bs", [16, 48, 64, 112, 256])
@pytest.mark.parametrize("hd", [64, 96, 128])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_append_is_exact(dt, hd, bs):
    """Ragged rows (one sequence without any), then single tokens that make scales grow, then a rollback."""
    pool = Pool(1, 5, -(-1200 // bs), 3, hd, bs)
    pool.upload()
    ref, rng, rope = pool.ref(), pool.rng, rope_table(1200, hd)
    pos = np.array([0, 5, bs - 1, 2 * bs, 37])
    for counts, scale in (([3, 33, 2 * bs + 1, 0, 1], 1.0), ([1] * 5, 40.0), ([2, 1, 0, 5, 17], 1e-3), ([1] * 5, 3e4)):
        n = sum(counts)
        k, v = (rng.standard_normal((n, 3, hd)) * scale * 2.0 ** rng.integers(-3, 3, (n, 3, 1)) for _ in range(2))
        append_both(pool, ref, dt, counts, pos, k, v, rope, rng.standard_normal((n, 9, hd)))
        pos = pos + np.array(counts)
    append_both(pool, ref, dt, [2] * 5, np.maximum(pos - 3, 0), rng.standard_normal((10, 3, hd)), rng.standard_normal((10, 3, hd)))
    same_cache(pool.kv, ref)


def test_append_odd_values():
    """NaN, infinities, zeros, subnormals, the largest floats: NaN codes where not finite, the block's scale from the rest."""
    pool = Pool(2, 4, 2, 2, 64, 16)
    pool.upload()
    ref = pool.ref()
    x = pool.rng.standard_normal((12, 2, 64)).astype(np.float32)
    x[0, 0, 3], x[1, 1, 5], x[1, 0, 7] = np.nan, np.inf, -np.inf
    x[3:6] = 0.0
    x[6:9] *= np.float32(1e-41)
    x[9] *= np.float32(1e38)
    x[10, :, ::2] = np.float32(3.4e38)
    append_both(pool, ref, "f32", [3, 3, 3, 3], [4, 0, 13, 14], x, x[::-1].copy())
    same_cache(pool.kv, ref)


def test_append_strided_rows_of_a_padded_batch():
    """k, v, q as parts of one projection; q turned in place; rows behind the last sequence stay as they were."""
    pool = Pool(3, 2, 4, 2, 96, 16)
    kv, ref, rope = pool.upload(), pool.ref(), rope_table(64, 96)
    x = torch.randn(9, 10, 96, device="cuda").bfloat16()
    was = x.clone()
    q, k, v = x[:, :6], x[:, 6:8], x[:, 8:]
    kv8_append(kv, k, v, i32([1, 4, 6]), i32([15, 30]), rope=torch.tensor(rope).cuda(), q=q, q_out=q)
    for s, (r, p) in enumerate(((slice(1, 4), 15), (slice(4, 6), 30))):
        n = r.stop - r.start
        f = was[r].float().cpu().numpy()
        t = kv8_ref.rotate(f[:, :8], rope[p:p + n])
        ref.append(0, pool.table[s], p, t[:, 6:])
        ref.append(1, pool.table[s], p, f[:, 8:])
        assert torch.equal(x[r, :6].cpu(), torch.tensor(t[:, :6]).bfloat16())
    same_cache(kv, ref)
    assert torch.equal(x[0], was[0]) and torch.equal(x[6:], was[6:]) and torch.equal(x[:, 6:], was[:, 6:])


def test_append_out_of_range_is_left_out():
    """Positions past the table or the rotation table, block ids outside the pool, negative positions, rows out of order: error
    bits, everything else written."""
    pool = Pool(4, 5, 2, 1, 64, 16)
    pool.table[2, 0] = 999
    kv, ref = pool.upload(), pool.ref()
    x = np.random.default_rng(0).standard_normal((10, 1, 64)).astype(np.float32)
    err, d = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor(x).cuda()
    kv8_append(kv, d, d, i32([0, 4, 4, 6, 8, 10]), i32([30, 0, 0, -1, 3]), errors=err)
    for which in range(2):
        ref.append(which, pool.table[0], 30, x[:2])
        ref.append(which, pool.table[4], 3, x[8:10])
    same_cache(kv, ref)
    assert err.item() == 2
    err.zero_()
    rope = rope_table(8, 64)
    kv8_append(kv, d[:4], d[:4], i32([0, 4, 4, 4, 4, 4]), i32([6, 0, 0, 0, 0]), rope=torch.tensor(rope).cuda(), errors=err)
    ref.append(0, pool.table[0], 6, kv8_ref.rotate(x[:2], rope[6:8]))
    ref.append(1, pool.table[0], 6, x[:2])
    same_cache(kv, ref)
    assert err.item() == 8
    err.zero_()
    kv8_append(kv, d, d, i32([0, -3, 2, 20, 20, 20]), i32([0] * 5), errors=err)
    assert err.item() & 32


def attend_both(pool, dt, counts, lens, G, *, visible=None, own=None, scale=None, q=None, ws=None, see=None, n_rows=None):
    """Runs the call and compares every row and head."""
    kv, ref, rng, H, hd = pool.kv, pool.ref(), pool.rng, pool.H, pool.hd
    start = np.concatenate([[0], np.cumsum(counts)])
    n = n_rows or int(start[-1])
    qd = (torch.tensor(rng.standard_normal((n, H * G, hd))) if q is None else torch.tensor(q)).to(DT[dt]).cuda()
    out = torch.full((n, H * G, hd), 5.0, dtype=DT[dt], device="cuda")
    kw = {}
    if own is not None:
        oi = np.asarray(own)
        ok, ov = (torch.tensor(rng.standard_normal((max(1, oi.max() + 1), H, hd))).to(DT[dt]).cuda() for _ in range(2))
        kw = dict(own=i32(oi), own_k=ok, own_v=ov)
    ws = kv8_workspace(kv, qd) if ws is None else ws
    kv8_attention(kv, qd, i32(start), i32(lens), out, ws, visible=None if visible is None else i32(visible), scale=scale,
                  **kw)
    sc = 1.0 / np.sqrt(hd) if scale is None else scale
    many = n * G > 128 * len(counts)
    e_p = 2.0 ** -23 if dt == "f32" else 2.0 ** -8 if many else 2.0 ** -16
    h = 2.0 ** -24 if dt == "f32" else 2.0 ** -8
    got, qf = out.double().cpu().numpy(), qd.double().cpu().numpy()
    for s, c in enumerate(counts):
        L = max(0, lens[s])
        K, V = (ref.values(w, pool.table[s], L) for w in range(2))
        for i in range(c):
            r = start[s] + i
            t = L - (c - 1 - i) if visible is None else visible[r]
            t = min(max(t, 0), L)
            for hq in range(H * G):
                k, v = K[:, hq // G], V[:, hq // G]
                o = None
                if own is not None and own[r] >= 0:
                    o = (ok[own[r], hq // G].double().cpu().numpy(), ov[own[r], hq // G].double().cpu().numpy())
                want = kv8_ref.attend(qf[r, hq], k, v, t, sc, o)
                ka, va = (k[:t], v[:t]) if o is None else (np.vstack([k[:t], o[0]]), np.vstack([v[:t], o[1]]))
                if not len(ka):
                    assert np.all(got[r, hq] == 0.0)
                    continue
                if not np.all(np.isfinite(ka)) or not np.all(np.isfinite(va)):
                    assert np.array_equal(np.isnan(got[r, hq]), np.isnan(want)), (s, i, hq)
                    if np.isnan(want).all():
                        continue
                    ok_d = ~np.isnan(want)
                    va, want, g = va[:, ok_d], want[ok_d], got[r, hq][ok_d]
                    ka = np.nan_to_num(ka)
                else:
                    g = got[r, hq]
                dz = U * (hd + 16) * sc * np.max(np.abs(ka) @ np.abs(qf[r, hq])) + 8 * U * np.max(np.abs(ka @ qf[r, hq])) * sc
                tol = np.max(np.abs(va)) * (2 * dz + e_p + 2 * U * (len(ka) + 128)) + h * np.abs(want)
                assert np.all(np.abs(g - want) <= tol), (s, i, hq, float(np.max(np.abs(g - want) / tol)))
    assert torch.all(out[int(start[-1]):] == 5.0)   # rows of no sequence
    return qd, out


@pytest.mark.parametrize("hd,bs", [(64, 16), (96, 16), (128, 16), (96, 48), (128, 256), (64, 112)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("H,G", [(3, 1), (2, 4), (1, 8)])
def test_decode_lengths(dt, hd, bs, H, G):
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 400, 1000]
    pool = Pool(5, len(lens), -(-1024 // bs), H, hd, bs)
    pool.upload()
    attend_both(pool, dt, [1] * len(lens), lens, G)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("counts,lens,G", [
    ([5], [701], 1), ([16], [16], 1), ([2, 16, 1, 7], [3, 900, 64, 7], 1), ([3, 0, 9], [2, 50, 1500], 4),
    ([100], [100], 1), ([130, 64], [130, 333], 2), ([300, 1, 40], [1000, 5, 64], 3), ([33], [20], 2), ([70, 257], [4000, 257], 1)])
@pytest.mark.parametrize("hd", [64, 96, 128])
def test_causal_chunks_and_prompts(dt, counts, lens, G, hd):
    """Short chunks and long ones; more rows than positions (the first rows see nothing)."""
    pool = Pool(6, len(counts), 256, 2, hd, 16)
    pool.upload()
    attend_both(pool, dt, counts, lens, G)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 40, 130])
def test_visible_and_own_keys(dt, n):
    """Rows that see none, some, more than there is; own keys for some, also where nothing else is seen."""
    pool = Pool(7, 3, 32, 2, 96, 16)
    pool.upload()
    rng = np.random.default_rng(8)
    vis = rng.integers(-3, 400, 3 * n)
    vis[::5] = 0
    own = np.where(rng.random(3 * n) < 0.5, rng.integers(0, 4, 3 * n), -1)
    own[0], own[-1] = 3, -1
    attend_both(pool, dt, [n] * 3, [350, 17, 0], 3, visible=vis, own=own, scale=0.17)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1024], [3, 300, 1024, 50, 12, 700, 800, 20]])
def test_dual_rows(dt, lens):
    """The decode step's form: the slow row sees all, the fast row all but the newest position and its own key."""
    B = len(lens)
    pool = Pool(9, B, 64, 4, 96, 16)
    pool.upload()
    vis = np.stack([lens, np.array(lens) - 1], 1).ravel()
    own = np.stack([-np.ones(B, int), np.arange(B)], 1).ravel()
    attend_both(pool, dt, [2] * B, lens, 1, visible=vis, own=own)


@pytest.mark.parametrize("n,G", [(4, 1), (60, 2), (100, 2)])
def test_what_is_not_seen_does_not_reach_a_row(n, G):
    """NaN codes behind the last position, and at positions that some rows of a chunk see and some do not, in keys and values."""
    pool = Pool(10, 2, 20, 2, 64, 16)
    lens = [200 + n, n + 3]
    for s, L in enumerate(lens):
        for w in range(2):
            for p in range(L, 20 * 16):
                pool.codes[w][pool.table[s, p // 16], :, p % 16] = 0x7f
        # one value of a position in the middle of the chunk; one key of a later one, of head 1
        p = L - n // 2
        pool.codes[1][pool.table[s, p // 16], 0, p % 16, 5] = 0xff
        pool.codes[0][pool.table[s, (L - 1) // 16], 1, (L - 1) % 16, 9] = 0x7f
    pool.upload()
    for dt in ("f32", "bf16"):
        attend_both(pool, dt, [n, n], lens, G)


def test_large_scores_and_scales():
    """Scores far apart (weights underflow), caches of very large and very small scales."""
    for lo, hi in ((-3, 3), (30, 36), (-60, -54)):
        pool = Pool(11, 2, 16, 2, 128, 16, scales=(lo, hi))
        pool.upload()
        q = pool.rng.standard_normal((2, 2, 128)) * 2.0 ** -lo * 4.0
        attend_both(pool, "f32", [1, 1], [256, 100], 1, q=q)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_many_short_sequences_and_padding(dt):
    rng = np.random.default_rng(12)
    lens = rng.integers(0, 60, 300)
    counts = rng.integers(0, 3, 300)
    pool = Pool(13, 300, 4, 1, 64, 16)
    pool.upload()
    attend_both(pool, dt, counts, lens, 2, n_rows=int(counts.sum()) + 5)


def test_one_long_context_is_split_and_joined():
    pool = Pool(14, 1, 1300, 1, 64, 16)
    pool.upload()
    for dt in ("bf16", "f32"):
        attend_both(pool, dt, [1], [20789], 2)
        attend_both(pool, dt, [20], [20789], 2)
        attend_both(pool, dt, [70], [20789], 2)


def test_blocks_outside_the_pool_are_left_out():
    """Their positions are not seen, the error bit is set; a table entry behind the last position is not looked at."""
    for n in (1, 40, 150):
        pool = Pool(15, 2, 8, 1, 64, 16)
        kept = pool.table.copy()
        pool.table[0, 2], pool.table[1, 7] = 5000, -7
        kv = pool.upload()
        q = torch.randn(2 * n, 1, 64, device="cuda")
        out, err = torch.zeros_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = kv8_workspace(kv, q)
        start = i32([0, n, 2 * n])
        vis = i32([100] * (2 * n))
        kv8_attention(kv, q, start, i32([0, 100]), out, ws, visible=vis, errors=err)
        assert err.item() == 0
        kv8_attention(kv, q, start, i32([100, 100]), out, ws, visible=vis, errors=err)
        assert err.item() == 2
        pool.table = kept
        K, V = (pool.ref().values(w, kept[0], 100)[:, 0] for w in range(2))
        there = np.r_[0:32, 48:100]
        for r in range(n):
            want = kv8_ref.attend(q[r, 0].double().cpu().numpy(), K[there], V[there], len(there), 0.125)
            assert np.allclose(out[r, 0].double().cpu().numpy(), want, atol=2e-5 * np.abs(V).max())
        # a length past the table, row starts that overlap: bits, and no result out of bounds
        err.zero_()
        kv8_attention(kv, q, start, i32([500, 3]), out, ws, errors=err)
        assert err.item() & 2
        err.zero_()
        kv8_attention(kv, q, i32([0, 4 * n, 2]), i32([9, 9]), out, ws, errors=err)
        assert err.item() & 32
        kv8_attention(kv, q, start, i32([100, 100]), out, ws, own=i32([7] * (2 * n)), own_k=q[:1], own_v=q[:1], errors=err)
        attend_both(pool_ok(pool), "f32", [n, n], [100, 90], 1, ws=ws)   # the workspace is as it was


def pool_ok(pool):
    pool.upload()
    return pool


def test_results_repeat_and_workspaces_serve_any_shape():
    pool = Pool(16, 4, 256, 2, 128, 16)
    pool.upload()
    big = kv8_workspace(pool.kv, torch.empty(600, 8, 128, device="cuda"))
    for counts, lens in (([1] * 4, [4000, 30, 2000, 1]), ([150] * 4, [4000, 200, 150, 3000]), ([2, 0, 0, 0], [4096, 1, 1, 1])):
        q, a = attend_both(pool, "bf16", counts, lens, 4, ws=big)
        for _ in range(3):
            b = torch.zeros_like(a)
            start = i32(np.concatenate([[0], np.cumsum(counts)]))
            kv8_attention(pool.kv, q, start, i32(lens), b, big)
            assert torch.equal(a[:sum(counts)], b[:sum(counts)])


def test_decoding_together_captured_and_replayed():
    """A prompt is appended and attended to, then decode steps (append, attend) replayed from a graph on another
    stream, with lengths that advance on the device; every step equals the eager one."""
    H, G, hd, B = 2, 3, 96, 3
    pool = Pool(17, B, 20, H, hd, 16)
    kv = pool.upload()
    rope = torch.tensor(rope_table(320, hd)).cuda()
    lens0 = [33, 7, 150]
    n = sum(lens0)
    g = torch.Generator(device="cuda").manual_seed(3)

    def rnd(*s):
        return torch.randn(*s, generator=g, device="cuda").bfloat16()

    q, k, v, out = rnd(n, H * G, hd), rnd(n, H, hd), rnd(n, H, hd), torch.zeros(n, H * G, hd, device="cuda").bfloat16()
    start = i32(np.concatenate([[0], np.cumsum(lens0)]))
    ws = kv8_workspace(kv, q)
    kv8_append(kv, k, v, start, i32([0] * B), rope=rope, q=q, q_out=q)
    kv8_attention(kv, q, start, i32(lens0), out, ws)
    pool.codes = [kv.k_pages.view(torch.uint8).cpu().numpy(), kv.v_pages.view(torch.uint8).cpu().numpy()]
    pool.scales = [kv.k_scales.double().cpu().numpy(), kv.v_scales.double().cpu().numpy()]
    ref = pool.ref()
    for s, L in enumerate(lens0):
        K, V = ref.values(0, pool.table[s], L), ref.values(1, pool.table[s], L)
        r = int(start[s + 1]) - 1
        for hq in range(H * G):
            want = kv8_ref.attend(q[r, hq].double().cpu().numpy(), K[:, hq // G], V[:, hq // G], L, hd ** -0.5)
            assert np.abs(out[r, hq].double().cpu().numpy() - want).max() < 2.0 ** -7 * np.abs(V).max()

    sq, sk, sv, so = rnd(B, H * G, hd), rnd(B, H, hd), rnd(B, H, hd), torch.zeros(B, H * G, hd, device="cuda").bfloat16()
    qr, pos, len_, one = torch.empty_like(sq), i32(lens0), i32(lens0) + 1, i32(range(B + 1))

    def step(kv, pos, len_, so, ws):
        kv8_append(kv, sk, sv, one, pos, rope=rope, q=sq, q_out=qr)
        kv8_attention(kv, qr, one, len_, so, ws)
        pos += 1
        len_ += 1

    other = KV8Pages(*(t.clone() for t in (kv.k_pages, kv.v_pages, kv.k_scales, kv.v_scales, kv.block_table)))
    p2, l2, o2, w2 = pos.clone(), len_.clone(), so.clone(), torch.zeros_like(ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(kv, pos, len_, so, ws)
        step(other, p2, l2, o2, w2)
        side.synchronize()
        assert torch.equal(so, o2)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(kv, pos, len_, so, ws)
    for i in range(20):
        for t in (sq, sk, sv):
            t.copy_(rnd(*t.shape) * 2.0 ** (i % 5))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(other, p2, l2, o2, w2)
        torch.cuda.synchronize()
        assert torch.equal(so, o2), i
        assert torch.equal(kv.k_pages.view(torch.uint8), other.k_pages.view(torch.uint8))
        assert torch.equal(kv.v_scales, other.v_scales)
    assert p2.tolist() == [L + 21 for L in lens0] and pos.tolist() == p2.tolist()


@pytest.mark.parametrize("n", [1, 40])
def test_broadcast_rows_and_empty_batches(n):
    """Both strides 0: every row and head reads the same vector; and empty batches enqueue nothing."""
    H, hd = 2, 64
    pool = Pool(19, 2, 4, H, hd, 16)
    kv, ref, rng = pool.upload(), pool.ref(), pool.rng
    x = torch.tensor(rng.standard_normal((1, 1, hd)), dtype=torch.float32, device="cuda").expand(n, H, hd)
    start = i32([0, n // 2, n])
    kv8_append(kv, x, x, start, i32([3, 9]))
    for s, (c, p) in enumerate(((n // 2, 3), (n - n // 2, 9))):
        if c:
            for which in range(2):
                ref.append(which, pool.table[s], p, np.broadcast_to(x[0].cpu().numpy(), (c, H, hd)))
    same_cache(kv, ref)
    none = torch.empty(0, H, hd, device="cuda")
    kv8_append(kv, none, none, i32([0, 0, 0]), i32([3, 9]), q=none, q_out=none)
    kv8_attention(kv, none, i32([0, 0, 0]), i32([3, 9]), none, kv8_workspace(kv, none))
    q, out = torch.randn(n, H, hd, device="cuda"), torch.zeros(n, H, hd, device="cuda")
    kv8_attention(kv, q, start, i32([20, 50]), out, kv8_workspace(kv, q), own=i32([-1] * n), own_k=none, own_v=none)
    same_cache(kv, ref)


@pytest.mark.parametrize("n,dt", [(2, "bf16"), (3, "f32"), (70, "bf16"), (200, "f32")])
def test_a_pool_beyond_32_bits(n, dt):
    """Blocks on both sides of 2^32 bytes (and 2^31): rows appended there, then attended to."""
    H, hd, bs, nb, L = 4, 128, 64, 140000, 1000 + n   # 32 KB a block and head set: 4.27 GiB of keys, as many of values
    pages = [torch.empty(nb, H, bs, hd, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.ones(nb, H, device="cuda") for _ in range(2)]
    near = [(1 << 31) // (H * bs * hd), (1 << 32) // (H * bs * hd)]
    want = [nb - 1, 0, near[0], near[0] - 1, near[1], near[1] - 1]
    blocks = np.array(want + [i * 8009 + 11 for i in range(-(-L // bs) - len(want))], dtype=np.int32)
    kv = KV8Pages(*pages, *scales, i32(blocks[None]))
    rng = np.random.default_rng(n)
    k, v = (torch.tensor(rng.standard_normal((L, H, hd))).to(DT[dt]).cuda() for _ in range(2))
    kv8_append(kv, k, v, i32([0, L]), i32([0]))
    small = Pool(20, 1, len(blocks), H, hd, bs)       # the same blocks, in order, as a pool of their own
    small.table = np.arange(len(blocks), dtype=np.int32)[None]
    small.codes = [np.zeros((len(blocks), H, bs, hd), np.uint8) for _ in range(2)]
    small.scales = [np.ones((len(blocks), H)) for _ in range(2)]
    small.upload()
    ref = small.ref()
    for which, x in enumerate((k, v)):
        ref.append(which, small.table[0], 0, x.float().cpu().numpy())
    for c, s, codes, exps in zip(pages, scales, ref.codes, ref.exps):
        got = c.view(torch.uint8)[torch.tensor(blocks, device="cuda").long()].cpu().numpy()
        for b in range(len(blocks)):
            m = min(bs, L - b * bs)
            assert np.array_equal(kv8_ref.CODE[got[b, :, :m]], kv8_ref.CODE[codes[b, :, :m]]), b
        assert np.array_equal(s[torch.tensor(blocks, device="cuda").long()].cpu().numpy(), 2.0 ** exps)
    small.codes, small.scales, small.kv = ref.codes, [2.0 ** e for e in ref.exps], kv
    attend_both(small, dt, [n], [L], 2)


def test_a_first_call_in_a_capture():
    """A program whose first call of the attention for many columns is captured: nothing of it waits for an eager one."""
    code = """
import torch, sys
sys.path.insert(0, {root!r})
from paper_2502_02040_amd import KV8Pages, kv8_attention, kv8_workspace
z = lambda *s: torch.randint(0, 120, s, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
one = lambda: torch.ones(64, 2, device="cuda")
kv = KV8Pages(z(64, 2, 16, 64), z(64, 2, 16, 64), one(), one(), torch.arange(64, dtype=torch.int32, device="cuda")[None].contiguous())
q, out = torch.randn(200, 4, 64, device="cuda").bfloat16(), torch.zeros(200, 4, 64, device="cuda").bfloat16()
start, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 200], [1000]))
ws = kv8_workspace(kv, q)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    kv8_attention(kv, q, start, lens, out, ws)
for _ in range(3):
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    a = out.clone()
    kv8_attention(kv, q, start, lens, out, ws)
    assert a.abs().sum() > 0 and torch.equal(a, out)
print("same")
"""
    root = str(pathlib.Path(__file__).resolve().parent.parent)
    r = subprocess.run([sys.executable, "-c", code.format(root=root)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]
