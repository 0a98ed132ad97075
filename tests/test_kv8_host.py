"""The 8-bit cache's operators refuse what they cannot take, before any device
work (no GPU needed: the pointers are never read)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2502_02040_amd import binding, kv8
from tests import kv8_ref

P = 1 << 20   # a 16-byte aligned address that no refused call touches


def _pages(**kw):
    d = dict(k_pages=P, v_pages=P, k_scales=P, v_scales=P, block_table_d=P, num_blocks=8, block_size=16,
             max_blocks_per_seq=4, n_kv_heads=2, head_dim=64)
    return kv8._Pages(**{**d, **kw})


def _rows(**kw):
    d = dict(n_seqs=1, n_rows=4, row_start_d=P, positions_d=P, dtype=binding.BF16, k=P, v=P, k_row=128, k_head=64,
             v_row=128, v_head=64)
    return kv8._Rows(**{**d, **kw})


def _query(**kw):
    d = dict(n_seqs=1, n_rows=4, row_start_d=P, lens_d=P, dtype=binding.BF16, n_heads=4, q=P, q_row=256, q_head=64,
             out=P, out_row=256, out_head=64)
    return kv8._Query(**{**d, **kw})


BAD_PAGES = [(dict(k_pages=None), -1), (dict(v_scales=None), -1), (dict(block_table_d=None), -1),
             (dict(k_pages=P + 8), -1), (dict(k_scales=P + 2), -1), (dict(block_size=8), -2), (dict(block_size=24), -2),
             (dict(block_size=272), -2), (dict(head_dim=80), -7), (dict(head_dim=256), -7), (dict(num_blocks=0), -2),
             (dict(n_kv_heads=0), -2), (dict(n_kv_heads=5000), -2), (dict(max_blocks_per_seq=0), -2),
             (dict(num_blocks=1 << 27), -2), (dict(max_blocks_per_seq=1 << 26), -2)]


@pytest.mark.parametrize("bad,status", BAD_PAGES)
def test_cache_descriptions_refused(bad, status):
    append, size, attention = kv8._lib()
    n = ctypes.c_size_t(0)
    assert append(_pages(**bad), _rows(), None) == status
    assert attention(_pages(**bad), _query(), P, 1 << 40, None) == status
    assert size(_pages(**bad), 1, 4, 4, n) == status
    assert binding.lib().m2r2_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(n_seqs=-1), -2), (dict(n_rows=-1), -2), (dict(n_rows=(1 << 26) + 1), -2), (dict(row_start_d=None), -1),
    (dict(positions_d=None), -1), (dict(positions_d=P + 2), -1), (dict(dtype=2), -3), (dict(k=None), -1),
    (dict(v=None), -1), (dict(k=P + 8), -1), (dict(k_row=132), -1), (dict(v_head=60), -1), (dict(k_row=-128), -2),
    (dict(rope_d=P + 4, rope_len=4), -1), (dict(rope_d=P, rope_len=0), -1), (dict(n_heads=3, q=P, q_out=P), -2),
    (dict(n_heads=4), -1), (dict(n_heads=4, q=P, q_out=None), -1), (dict(q=P), -1), (dict(err_d=P + 1), -1),
    (dict(n_heads=4, q=P, q_out=P, q_row=256, q_head=64, qo_row=512, qo_head=64), -1)])
def test_rows_refused(bad, status):
    assert kv8._lib()[0](_pages(), _rows(**bad), None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(n_seqs=-1), -2), (dict(lens_d=None), -1), (dict(row_start_d=P + 2), -1), (dict(visible_d=P + 1), -1),
    (dict(dtype=5), -3), (dict(n_heads=0), -2), (dict(n_heads=3), -2), (dict(q=None), -1), (dict(q=P + 2), -1),
    (dict(out=None), -1), (dict(out_row=260), -1), (dict(own_d=P), -2), (dict(own_d=P, n_own=1), -1),
    (dict(own_d=P, n_own=1, own_k=P, own_v=P + 4), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(n_rows=1 << 26, n_heads=64), -2)])
def test_queries_refused(bad, status):
    assert kv8._lib()[2](_pages(), _query(**bad), P, 1 << 62, None) == status


def test_missing_descriptors_and_small_workspaces():
    append, size, attention = kv8._lib()
    n = ctypes.c_size_t(0)
    assert append(None, _rows(), None) == -1 and append(_pages(), None, None) == -1
    assert attention(_pages(), None, P, 1 << 40, None) == -1
    assert size(_pages(), 1, 4, 4, None) == -1
    assert size(_pages(), 1, 4, 4, n) == 0 and n.value > 0
    assert attention(_pages(), _query(), P, n.value - 1, None) == -4
    assert attention(_pages(), _query(), None, n.value, None) == -1
    assert attention(_pages(), _query(), P + 16, n.value, None) == -1


def test_nothing_to_do_is_no_error():
    append, _, attention = kv8._lib()
    assert append(_pages(), _rows(n_rows=0), None) == 0
    assert append(_pages(), _rows(n_seqs=0), None) == 0
    assert attention(_pages(), _query(n_seqs=0), P, 1 << 40, None) == 0


def test_packed_descriptions_are_the_structures():
    """The binding's struct formats lay out what the ctypes structures do."""
    for fmt, kind in ((kv8._ROWS, kv8._Rows), (kv8._QUERY, kv8._Query)):
        values = [0.5 if t is ctypes.c_float else i + 1 for i, (_, t) in enumerate(kind._fields_)]
        got = kind.from_buffer_copy(fmt.pack(*values))
        assert ctypes.sizeof(kind) == fmt.size and [getattr(got, n) for n, _ in kind._fields_] == values
    assert bytes(_pages()) == bytes(kv8._Pages.from_buffer_copy(bytes(_pages())))


def test_empty_calls_need_no_arrays():
    """A step without rows or without sequences: torch's empty tensors have no address."""
    append, size, attention = kv8._lib()
    none = dict(row_start_d=P, k=None, v=None, q=None, q_out=None, n_heads=4)
    assert append(_pages(), _rows(n_rows=0, **none), None) == 0
    assert append(_pages(block_table_d=None), _rows(n_seqs=0, positions_d=None), None) == 0
    assert attention(_pages(), _query(n_rows=0, q=None, out=None), P, 1 << 40, None) == 0
    assert attention(_pages(block_table_d=None), _query(n_seqs=0, lens_d=None), P, 1 << 40, None) == 0
    n = ctypes.c_size_t(0)
    assert size(_pages(block_table_d=None), 0, 0, 4, n) == 0


@pytest.mark.parametrize("bad", [dict(out_row=0), dict(out_head=0), dict(out_row=128), dict(out_head=128, out_row=256),
                                 dict(out_row=64, out_head=128)])
def test_overlapping_results_refused(bad):
    assert kv8._lib()[2](_pages(), _query(**bad), P, 1 << 40, None) == -1
    turned = {k.replace("out", "qo"): x for k, x in bad.items()}
    d = dict(n_heads=4, q=2 * P, q_out=P, q_row=256, q_head=64, qo_row=256, qo_head=64)
    assert kv8._lib()[0](_pages(), _rows(**{**d, **turned}), None) == -1


def test_more_workgroups_than_a_launch_holds():
    """n_rows and heads within their own limits, refused together (2^32 threads)."""
    append, size, _ = kv8._lib()
    n = ctypes.c_size_t(0)
    big = _pages(n_kv_heads=64)
    assert size(big, 1, 1 << 25, 64, n) == -2 and n.value == 0
    assert append(big, _rows(n_rows=1 << 25, k_row=4096, v_row=4096), None) == -2
    assert size(_pages(n_kv_heads=8), 1, 1 << 20, 32, n) == 0   # a million rows are not too many
    assert append(_pages(), _rows(k_row=(1 << 36) + 8), None) == -2


def test_workspace_grows_with_the_call():
    _, size, _ = kv8._lib()
    got = []
    for seqs, rows in ((1, 1), (1, 16), (4, 64), (4, 4096)):
        n = ctypes.c_size_t(0)
        assert size(_pages(max_blocks_per_seq=4096), seqs, rows, 8, n) == 0
        got.append(n.value)
    assert got[0] < got[1] and max(got) < 1 << 30


def _tensors(dev="cpu", bs=16, hd=64, H=2):
    k = torch.zeros(4, H, bs, hd, dtype=torch.float8_e4m3fn, device=dev)
    s = torch.ones(4, H, device=dev)
    return k, torch.zeros_like(k), s, s.clone(), torch.zeros(1, 4, dtype=torch.int32, device=dev)


def test_binding_refuses_wrong_tensors():
    k, v, ks, vs, bt = _tensors()
    kv = kv8.KV8Pages(k, v, ks, vs, bt)
    for args in ((k.view(torch.uint8), v, ks, vs, bt), (k.transpose(1, 2), v, ks, vs, bt), (k, v[:2], ks, vs, bt),
                 (k, v, ks.double(), vs, bt), (k, v, ks, vs, bt.long()), (k, v, ks[:, :1], vs, bt)):
        with pytest.raises(ValueError):
            kv8.KV8Pages(*args)
    i32 = dict(dtype=torch.int32)
    row, start, pos = torch.zeros(3, 2, 64), torch.zeros(2, **i32), torch.zeros(1, **i32)
    for a in ((row[:, :, :32], row, start, pos), (row, row.bfloat16(), start, pos), (row, row[:2], start, pos),
              (row, row, start[:1], pos), (row, row, start.long(), pos), (row.half(), row.half(), start, pos),
              (row, row, start, pos)):   # (the last: not on a GPU)
        with pytest.raises(ValueError):
            kv8.kv8_append(kv, *a)
    with pytest.raises(ValueError):
        kv8.kv8_append(kv, row, row, start, pos, q=row)
    with pytest.raises(ValueError):
        kv8.kv8_append(kv, row, row, start, pos, rope=torch.zeros(4, 32))
    with pytest.raises(ValueError):
        kv8.kv8_attention(kv, row, start, pos, row[:2], torch.zeros(4, dtype=torch.uint8))
    ws, own = torch.zeros(4, dtype=torch.uint8), torch.zeros(3, **i32)
    for kw in (dict(own=own), dict(own_k=row, own_v=row), dict(scale=0.0), dict(scale=float("nan"))):
        with pytest.raises(ValueError):
            kv8.kv8_attention(kv, row, start, pos, torch.zeros_like(row), ws, **kw)
    with pytest.raises(ValueError):
        kv8.kv8_attention(kv, row[0], start, pos, row[0], ws)
    with pytest.raises(binding.M2R2Error):
        kv8.kv8_workspace(kv, torch.zeros(2, 3, 64))


# ---- the reference itself --------------------------------------------------------------

def test_reference_codes_are_torchs():
    assert np.array_equal(kv8_ref.CODE, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(),
                          equal_nan=True)
    x = torch.cat([torch.randn(20000) * 40, torch.randn(20000) * 0.01, torch.tensor([0.0, -0.0, 448.0, -448.0, 2.0 ** -10])])
    mids = torch.tensor((kv8_ref.CODE[:126] + kv8_ref.CODE[1:127]) / 2, dtype=torch.float32)
    x = torch.cat([x.clamp(-448, 448), mids, -mids])
    assert np.array_equal(kv8_ref.encode(x.double().numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_reference_growing_scale_requantises():
    """Three appends into one block: values stay within half a code step of what was appended, at the scale they ended up with."""
    rng = np.random.default_rng(3)
    c = kv8_ref.Cache([np.zeros((1, 1, 16, 64))] * 2, [np.ones((1, 1))] * 2)
    rows = [rng.standard_normal((5, 1, 64)) * s for s in (1.0, 30.0, 0.1)]
    for i, r in enumerate(rows):
        c.append(0, np.array([0]), 5 * i, r)
    got, want = c.values(0, np.array([0]), 15)[:, 0], np.concatenate(rows)[:, 0]
    scale = 2.0 ** c.exps[0][0, 0]
    # one rounding to 4 significant bits (2^-4), and one to the grown scale's subnormal step
    assert np.all(np.abs(got - want) <= np.abs(want) * 2.0 ** -4 + 2 * scale * 2.0 ** -10)
