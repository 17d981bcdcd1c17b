"""Host-side refusals of the e4m3 cache's calls, of fork and of compact: every call here
fails validation before anything is enqueued (pointers are never dereferenced); and the
references that the GPU tests go by, against hand-made cases."""
import numpy as np
import pytest

import cache_f8_reference as ref
import paper_2601_07892_amd as sh

L = sh.lib
FAKE = 0x10000
I, S, A, B = sh.SHERRY_E_INVALID, sh.SHERRY_E_SHAPE, sh.SHERRY_E_ALIGN, sh.SHERRY_E_BUFSIZE


def _set(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _cache(**kw):
    c = sh.sherry_cache_desc()
    c.k = c.v = c.table = c.k_scale = c.v_scale = FAKE
    c.type, c.pages, c.kv_heads, c.page_size, c.head_dim, c.batch, c.table_width = sh.SHERRY_F8, 4, 2, 16, 64, 1, 4
    return _set(c, kw)


def _extend(**kw):
    d = sh.sherry_extend_desc()
    d.q = d.k = d.v = d.q_out = d.first = d.length = d.pos = d.cos = d.sin = FAKE
    d.tokens, d.heads, d.rope_rows, d.rot_dim = 3, 8, 10, 64
    return _set(d, kw)


def _tokens(**kw):
    d = sh.sherry_attend_tokens_desc()
    d.q = d.out = d.first = d.length = d.workspace = FAKE
    d.workspace_bytes, d.tokens, d.heads, d.scale = 1 << 40, 3, 8, 0.125
    return _set(d, kw)


def _fork(**kw):
    d = sh.sherry_fork_desc()
    d.parent = d.length = d.add = d.from_row = FAKE
    d.table_out = d.length_out = d.missing = d.workspace = FAKE + 64
    d.workspace_bytes, d.layers = 1 << 40, 1
    return _set(d, kw)


def _compact(**kw):
    d = sh.sherry_compact_desc()
    d.length = d.table_out = d.moved = d.live = d.workspace = FAKE
    d.workspace_bytes, d.layers = 1 << 40, 1
    return _set(d, kw)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), I), (dict(table=None), I), (dict(k_scale=None), I), (dict(v_scale=None), I), (dict(type=5), I),
    (dict(head_dim=72), S), (dict(page_stride=2 * 16 * 64 + 8), S), (dict(pages=0), S), (dict(batch=0), S),
    (dict(k=FAKE + 8), A), (dict(k_scale=FAKE + 4), A), (dict(table=FAKE + 2), A)])
def test_caches_refused(kw, status):
    c = _cache(**kw)
    assert L.sherry_cache_extend(c, _extend(), None) == status
    assert L.sherry_cache_attend_tokens(c, _tokens(), None) == status
    assert L.sherry_cache_attend_tokens_workspace(c, _tokens()) == 0
    if "type" not in kw:
        assert L.sherry_cache_fork(c, _fork(), None) == status
        assert L.sherry_cache_compact(c, _compact(), None) == status
        assert L.sherry_cache_fork_workspace(c, _fork()) == 0
        assert L.sherry_cache_compact_workspace(c, _compact()) == 0


def test_calls_that_another_cache_takes():
    """append and evict have no e4m3 form; extend and attend_tokens no other."""
    a = sh.sherry_append_desc()
    a.k = a.v = a.seq = a.slot = a.pos = FAKE
    a.tokens = 1
    assert L.sherry_cache_append(_cache(), a, None) == I
    e = sh.sherry_evict_desc()
    e.length, e.weight, e.length_out, e.kept = FAKE, FAKE, FAKE + 64, FAKE
    e.row_stride, e.out_stride, e.keep = 64, 32, 32
    assert L.sherry_cache_evict(_cache(), e, None) == I
    for kind in (sh.SHERRY_BF16, sh.SHERRY_F16):
        c = _cache(type=kind, k_scale=None, v_scale=None)
        assert L.sherry_cache_extend(c, _extend(), None) == I
        assert L.sherry_cache_attend_tokens(c, _tokens(), None) == I
    c = _cache(type=sh.SHERRY_I8)
    assert L.sherry_cache_extend(c, _extend(), None) == I
    assert L.sherry_cache_attend_tokens(c, _tokens(), None) == I


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), I), (dict(v=None), I), (dict(first=None), I), (dict(length=None), I), (dict(q=None), I),
    (dict(q_out=None), I), (dict(cos=None), I), (dict(sin=None), I), (dict(type=sh.SHERRY_I8), I),
    (dict(type=sh.SHERRY_F8), I), (dict(pairing=2), I), (dict(tokens=0), S), (dict(tokens=(1 << 24) + 1), S),
    (dict(heads=0), S), (dict(rope_rows=0), S), (dict(rot_dim=33), S), (dict(rot_dim=66), S), (dict(k_stride=127), S),
    (dict(v_stride=-1), S), (dict(q_stride=511), S), (dict(q_out_stride=8), S), (dict(q_stride=600), S),
    (dict(tokens=1 << 24, heads=1 << 20), S), (dict(k=FAKE + 2), A), (dict(q=FAKE + 1, q_out=FAKE), A),
    (dict(type=sh.SHERRY_F16, v=FAKE + 1), A), (dict(first=FAKE + 2), A), (dict(length=FAKE + 1), A),
    (dict(pos=FAKE + 2), A), (dict(cos=FAKE + 2), A)])
def test_extend_refused(kw, status):
    assert L.sherry_cache_extend(_cache(), _extend(**kw), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), I), (dict(out=None), I), (dict(first=None), I), (dict(length=None), I), (dict(workspace=None), I),
    (dict(type=3), I), (dict(window=-1), I), (dict(scale=float("nan")), I), (dict(scale=float("-inf")), I),
    (dict(tokens=0), S), (dict(tokens=(1 << 24) + 1), S), (dict(heads=1), S), (dict(heads=7), S), (dict(heads=2 * 257), S),
    (dict(tokens=1 << 24, heads=256), S), (dict(q_stride=508), S), (dict(q_stride=516), S), (dict(out_stride=504), S),
    (dict(mask=FAKE, mask_stride=63), S), (dict(q=FAKE + 8), A), (dict(out=FAKE + 4), A), (dict(workspace=FAKE + 8), A),
    (dict(first=FAKE + 2), A), (dict(length=FAKE + 2), A), (dict(workspace_bytes=100), B)])
def test_attend_tokens_refused(kw, status):
    assert L.sherry_cache_attend_tokens(_cache(), _tokens(**kw), None) == status


def test_null_descriptors():
    assert L.sherry_cache_extend(_cache(), None, None) == I
    assert L.sherry_cache_attend_tokens(_cache(), None, None) == I
    assert L.sherry_cache_fork(_cache(), None, None) == I
    assert L.sherry_cache_compact(_cache(), None, None) == I
    assert L.sherry_cache_fork(None, _fork(), None) == I


LAYERS = [
    (dict(layers=0), S), (dict(layers=65536), S), (dict(layers=2), S), (dict(layers=2, layer_stride=4 * 2048 - 16), S),
    (dict(layers=2, layer_stride=4 * 2048 + 8, scale_layer_stride=8), S),
    (dict(layers=2, layer_stride=4 * 2048, scale_layer_stride=7), S), (dict(workspace=None), I),
    (dict(length=None), I), (dict(table_out=None), I), (dict(workspace=FAKE + 4), A), (dict(length=FAKE + 1), A),
    (dict(table_out=FAKE + 2), A), (dict(workspace_bytes=10), B)]


@pytest.mark.parametrize("kw,status", LAYERS + [
    (dict(length_out=None), I), (dict(missing=None), I), (dict(length_out=FAKE), I), (dict(table_out=FAKE), I),
    (dict(parent=FAKE + 2), A), (dict(add=FAKE + 2), A), (dict(from_row=FAKE + 2), A), (dict(missing=FAKE + 2), A),
    (dict(length_out=FAKE + 2), A)])
def test_fork_refused(kw, status):
    assert L.sherry_cache_fork(_cache(), _fork(**kw), None) == status


@pytest.mark.parametrize("kw,status", LAYERS + [(dict(live=None), I), (dict(live=FAKE + 2), A), (dict(moved=FAKE + 2), A)])
def test_compact_refused(kw, status):
    assert L.sherry_cache_compact(_cache(), _compact(**kw), None) == status


def test_tables_past_31_bits_refused():
    c = _cache(batch=65535, table_width=1 << 20, page_size=1)
    assert L.sherry_cache_fork(c, _fork(), None) == S
    assert L.sherry_cache_compact(c, _compact(), None) == S


def test_workspaces_grow_with_the_pool():
    sizes = [sh.sherry_cache_fork_workspace(_cache(pages=p), _fork()) for p in (4, 4000, 4_000_000)]
    assert 0 < sizes[0] <= sizes[1] < sizes[2]
    assert 0 < sh.sherry_cache_compact_workspace(_cache(), _compact())
    one = sh.sherry_cache_attend_tokens_workspace(_cache(), _tokens(tokens=1))
    many = sh.sherry_cache_attend_tokens_workspace(_cache(table_width=1000), _tokens(tokens=1000))
    assert 0 < one < many <= 1 << 28


# ---- the references ---------------------------------------------------------------

def test_codes_are_e4m3():
    import torch
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.VALUES, want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.02, 0.02, 4001), ref._MIDDLE, -ref._MIDDLE])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x.astype(np.float64)), want)


def test_powers():
    assert [ref.power_of(np.float32([x])) for x in (0, 448, 448.00003, 1, 1.75, 1.76, 1e-44, np.inf)] == \
        [-100, 0, 1, -8, -8, -7, -100, -100]


def test_fork_reference_by_hand():
    # two sequences share page 0; the first goes on, the second goes on from the first
    table = np.array([[0, 1], [0, 2]], np.int32)
    out, n, missing, copies = ref.fork_plain(table, [20, 20], 6, 16, [0, 0], [1, 1], None)
    assert out.tolist() == [[0, 2], [0, 1]] and n.tolist() == [20, 20] and copies == [(1, 2)] and missing == 0
    # the second ends: its page is given out again
    out, n, missing, copies = ref.fork_plain(table, [20, 20], 3, 16, [0, -1], [20, 0], None)
    assert missing == 0 and out.tolist() == [[0, 1], [-1, -1]] and n.tolist() == [20, 0] and not copies
    # both write all of it: the first needs two pages, one is free
    assert ref.fork_plain(table, [20, 20], 3, 16, [0, 0], [1, 1], [0, 0])[2] == 1


def test_compact_reference_by_hand():
    out, moved, live, copies = ref.compact_plain(np.array([[5, 1], [3, 7]], np.int32), [20, 3], 8, 16)
    assert live == 3 and copies == [(3, 0), (5, 2)]
    assert out.tolist() == [[2, 1], [0, -1]] and moved.tolist() == [-1, 1, -1, 0, -1, 2, -1, -1]
