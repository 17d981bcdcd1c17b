"""Host-side refusals of the products with an epilogue and of the paged cache:
every call here fails validation before anything is enqueued (pointers are
never dereferenced)."""
import ctypes

import pytest

import paper_2601_07892_amd as sh

L = sh.lib
FAKE = 0x10000


def _cache(**kw):
    c = sh.sherry_cache_desc()
    c.k = c.v = c.table = FAKE
    c.type, c.pages, c.kv_heads, c.page_size, c.head_dim, c.batch, c.table_width = sh.SHERRY_BF16, 4, 2, 16, 64, 1, 4
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _append(**kw):
    d = sh.sherry_append_desc()
    d.q = d.k = d.v = d.q_out = d.seq = d.slot = d.pos = d.cos = d.sin = d.weight = d.position = FAKE
    d.row_stride, d.tokens, d.heads, d.rope_rows, d.rot_dim = 64, 3, 8, 10, 64
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _attend(**kw):
    d = sh.sherry_attend_desc()
    d.q = d.out = d.length = d.workspace = FAKE
    d.workspace_bytes, d.heads, d.scale = 1 << 40, 8, 0.125
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _evict(**kw):
    d = sh.sherry_evict_desc()
    d.length, d.length_out = FAKE, FAKE + 64
    d.weight = d.position = d.recent_from = d.kept = d.weight_out = d.position_out = FAKE
    d.row_stride, d.out_stride, d.keep = 64, 32, 32
    for k, v in kw.items():
        setattr(d, k, v)
    return d


I, S, A = sh.SHERRY_E_INVALID, sh.SHERRY_E_SHAPE, sh.SHERRY_E_ALIGN
BAD_CACHES = [
    (dict(k=None), I), (dict(v=None), I), (dict(table=None), I), (dict(type=sh.SHERRY_F32), I), (dict(type=9), I),
    (dict(type=-1), I), (dict(k_scale=FAKE), I), (dict(type=sh.SHERRY_I8), I),
    (dict(type=sh.SHERRY_I8, k_scale=FAKE), I), (dict(type=sh.SHERRY_I8, k_scale=FAKE, v_scale=FAKE, head_dim=72), S),
    (dict(pages=0), S), (dict(kv_heads=0), S), (dict(kv_heads=5000), S), (dict(page_size=0), S), (dict(head_dim=0), S),
    (dict(head_dim=12), S), (dict(head_dim=264), S), (dict(batch=0), S), (dict(batch=1 << 20), S),
    (dict(table_width=0), S), (dict(table_width=1 << 27), S), (dict(page_stride=2 * 16 * 64 - 8), S),
    (dict(page_stride=2 * 16 * 64 + 4), S), (dict(k=FAKE + 8), A), (dict(v=FAKE + 2), A), (dict(table=FAKE + 2), A),
    (dict(type=sh.SHERRY_I8, k_scale=FAKE + 4, v_scale=FAKE), A),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_refused(kw, status):
    c = _cache(**kw)
    assert L.sherry_cache_append(c, _append(), None) == status
    assert L.sherry_cache_attend(c, _attend(), None) == status
    assert L.sherry_cache_evict(c, _evict(), None) == status
    assert L.sherry_cache_attend_workspace(c, _attend()) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), I), (dict(v=None), I), (dict(seq=None), I), (dict(slot=None), I), (dict(pos=None), I),
    (dict(q=None), I), (dict(q_out=None), I), (dict(cos=None), I), (dict(sin=None), I), (dict(type=sh.SHERRY_I8), I),
    (dict(pairing=2), I), (dict(tokens=0), S), (dict(tokens=(1 << 24) + 1), S), (dict(heads=0), S),
    (dict(rope_rows=0), S), (dict(rot_dim=0), S), (dict(rot_dim=33), S), (dict(rot_dim=66), S), (dict(row_stride=63), S),
    (dict(k_stride=127), S), (dict(v_stride=-1), S), (dict(q_stride=511), S), (dict(q_out_stride=8), S),
    (dict(k=FAKE + 2), A), (dict(q=FAKE + 1), A), (dict(type=sh.SHERRY_F16, v=FAKE + 1), A), (dict(pos=FAKE + 2), A),
    (dict(weight=FAKE + 1), A), (dict(cos=FAKE + 2), A)])
def test_append_refused(kw, status):
    assert L.sherry_cache_append(_cache(), _append(**kw), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), I), (dict(out=None), I), (dict(length=None), I), (dict(workspace=None), I), (dict(type=3), I),
    (dict(window=-1), I), (dict(scale=float("nan")), I), (dict(scale=float("inf")), I),
    (dict(window=4, position=FAKE, row_stride=64), I), (dict(heads=1), S), (dict(heads=7), S), (dict(heads=2 * 257), S),
    (dict(q_stride=508), S), (dict(q_stride=516), S), (dict(out_stride=504), S), (dict(mask=FAKE, mask_stride=63), S),
    (dict(weight=FAKE, row_stride=63), S), (dict(position=FAKE), S), (dict(q=FAKE + 8), A), (dict(out=FAKE + 4), A),
    (dict(workspace=FAKE + 8), A), (dict(length=FAKE + 1), A), (dict(weight=FAKE + 2, row_stride=64), A),
    (dict(workspace_bytes=100), sh.SHERRY_E_BUFSIZE)])
def test_attend_refused(kw, status):
    assert L.sherry_cache_attend(_cache(), _attend(**kw), None) == status


def test_attend_rows_refused():
    """More rows in all than are counted."""
    c = _cache(batch=128, page_size=1 << 20, table_width=1 << 10)
    assert L.sherry_cache_attend(c, _attend(), None) == S
    assert L.sherry_cache_attend_workspace(c, _attend()) == 0
    assert sh.sherry_cache_attend_workspace(_cache(batch=32, page_size=1 << 20, table_width=1 << 10), _attend()) > 0


def test_attend_workspace():
    """Grows with the splits and, for weight, with the scores; exactly that much
    is enough for the call (one byte less is refused)."""
    c, d = _cache(batch=3, table_width=100), _attend()
    plain = sh.sherry_cache_attend_workspace(c, d)
    assert plain > 0
    w = sh.sherry_cache_attend_workspace(c, _attend(weight=FAKE, row_stride=1600))
    assert w - plain == 3 * 8 * 1600 * 4
    d.workspace_bytes = plain - 1
    assert L.sherry_cache_attend(c, d, None) == sh.SHERRY_E_BUFSIZE
    assert sh.sherry_cache_attend_workspace(c, _attend(q=None, workspace=None)) == plain


@pytest.mark.parametrize("kw,status", [
    (dict(length=None), I), (dict(weight=None), I), (dict(length_out=None), I), (dict(kept=None), I),
    (dict(length_out=FAKE), I), (dict(keep=0), S), (dict(keep=-1), S), (dict(out_stride=31), S), (dict(row_stride=63), S),
    (dict(kept=FAKE + 1), A), (dict(weight=FAKE + 2), A), (dict(position_out=FAKE + 2), A)])
def test_evict_refused(kw, status):
    assert L.sherry_cache_evict(_cache(), _evict(**kw), None) == status


def test_null_descriptors_refused():
    assert L.sherry_cache_append(None, _append(), None) == I
    assert L.sherry_cache_append(_cache(), None, None) == I
    assert L.sherry_cache_attend(_cache(), None, None) == I
    assert L.sherry_cache_evict(_cache(), None, None) == I
    assert L.sherry_cache_attend_workspace(None, None) == 0
    with pytest.raises(sh.SherryError) as e:
        sh.sherry_cache_append(_cache(pages=0), _append(), stream=0)
    assert e.value.status == S


def _epi(**kw):
    e = sh.sherry_epilogue()
    for k, v in kw.items():
        setattr(e, k, v)
    return e


@pytest.mark.parametrize("epi,scales,status", [
    (None, (None, None), I), (_epi(act=6), (None, None), I), (_epi(act=-1), (None, None), I),
    (_epi(), (FAKE, FAKE), I), (_epi(gate=FAKE, gate_stride=63), (None, None), S),
    (_epi(residual=FAKE, residual_stride=-64), (None, None), S), (_epi(bias=FAKE + 1), (None, None), A),
    (_epi(gate=FAKE + 2), (None, None), A), (_epi(residual=FAKE + 2), (None, None), A), (_epi(), (FAKE + 2, None), A),
    (_epi(), (None, FAKE + 1), A)])
@pytest.mark.parametrize("m", [1, 40])
def test_epilogues_refused(epi, scales, status, m):
    assert L.sherry_gemm_epilogue(FAKE, FAKE, FAKE, 1.0, *scales, epi, FAKE, m, 64, 128, None) == status
    if m == 1:
        assert L.sherry_gemv_f32_epilogue(FAKE, FAKE, None, 1.0, *scales, epi, FAKE, 64, 128, None) == status


@pytest.mark.parametrize("m", [1, 40])
def test_epilogue_products_refused(m):
    e = _epi()
    f = L.sherry_gemm_epilogue
    assert f(None, FAKE, FAKE, 1.0, None, None, e, FAKE, m, 64, 128, None) == I
    assert f(FAKE, FAKE, None, 1.0, None, None, e, FAKE, m, 64, 128, None) == I
    assert f(FAKE, FAKE, FAKE, 1.0, None, None, e, None, m, 64, 128, None) == I
    assert f(FAKE, FAKE, FAKE, 1.0, None, None, e, FAKE, 0, 64, 128, None) == S
    assert f(FAKE, FAKE, FAKE, 1.0, None, None, e, FAKE, m, 64, 126, None) == S
    assert f(FAKE + 8, FAKE, FAKE, 1.0, None, None, e, FAKE, m, 64, 128, None) == A
    assert f(FAKE, FAKE + 2, FAKE, 1.0, None, None, e, FAKE, m, 64, 128, None) == A
    g = L.sherry_gemv_f32_epilogue
    assert g(FAKE, FAKE, None, 1.0, None, None, e, FAKE, 64, sh.SHERRY_FUSED_MAX_K + 4, None) == S
    assert g(FAKE, FAKE + 4, None, 1.0, None, None, e, FAKE, 64, 128, None) == A
    assert g(FAKE, None, None, 1.0, None, None, e, FAKE, 64, 128, None) == I


def test_descriptor_sizes():
    """The layouts of the header (checked there against the C side)."""
    for cls, n in ((sh.sherry_epilogue, 48), (sh.sherry_cache_desc, 80), (sh.sherry_append_desc, 152),
                   (sh.sherry_attend_desc, 120), (sh.sherry_evict_desc, 88)):
        assert ctypes.sizeof(cls) == n


@pytest.mark.parametrize("strides", [(600, 0), (0, 600), (600, 520), (512, 600)])
def test_append_in_place_with_other_strides_refused(strides):
    """q_out = q and rows that lie elsewhere: a token's output would be another
    token's unread row."""
    d = _append(q_stride=strides[0], q_out_stride=strides[1])
    assert L.sherry_cache_append(_cache(), d, None) == S
    d.q_out = FAKE + 4 * 600 * 3  # apart: passes that check (and fails a later one)
    d.pos = FAKE + 2
    assert L.sherry_cache_append(_cache(), d, None) == A
    d = _append(q_stride=strides[0], q_out_stride=strides[1], tokens=1, pos=FAKE + 2)  # one row: no other
    assert L.sherry_cache_append(_cache(), d, None) == A
    for same in ((0, 512), (512, 0), (600, 600)):
        d = _append(q_stride=same[0], q_out_stride=same[1], pos=FAKE + 2)
        assert L.sherry_cache_append(_cache(), d, None) == A


def test_limits_of_the_header():
    """The largest values that the header names pass, the next ones do not."""
    def size(cache, **kw):
        return L.sherry_cache_attend_workspace(_cache(**cache), _attend(**kw))
    assert size(dict(batch=65535)) > 0 and size(dict(batch=65536)) == 0
    assert size(dict(kv_heads=4096), heads=4096) > 0 and size(dict(kv_heads=4097), heads=4097) == 0
    assert size({}, heads=2 * 256) > 0 and size({}, heads=2 * 257) == 0
    assert size(dict(head_dim=256)) > 0 and size(dict(head_dim=264)) == 0
    top = dict(page_size=1 << 20, table_width=1 << 10)
    assert size(top) > 0 and size(dict(top, table_width=(1 << 10) + 1)) == 0
    late = dict(pos=FAKE + 2)  # fails the last of the checks
    assert L.sherry_cache_append(_cache(batch=65535), _append(**late), None) == A
    assert L.sherry_cache_append(_cache(), _append(heads=256 * 4096, tokens=1, **late), None) == A
    assert L.sherry_cache_append(_cache(), _append(heads=256 * 4096 + 1, tokens=1, **late), None) == S
    assert L.sherry_cache_evict(_cache(batch=65535), _evict(kept=FAKE + 1), None) == A


def test_launches_of_more_threads_than_a_grid_holds_refused():
    """2^32 - 1 threads, 256 a workgroup (1024 in eviction's selection): calls at
    the limit pass to a later check, the next ones are refused before anything is
    enqueued."""
    late = dict(pos=FAKE + 2)

    def append(tokens, heads, **cache):
        return L.sherry_cache_append(_cache(**cache), _append(tokens=tokens, heads=heads, **late), None)
    top = (1 << 24) - 1  # workgroups
    assert append(top, 12) == A and append(top + 1, 12) == S  # 16 rows of 64 values: one a token
    assert append(top // 2, 13) == A and append(top // 2 + 1, 13) == S
    assert append(top // 2, 12, head_dim=128) == A and append(top // 2 + 1, 12, head_dim=128) == S
    assert append(top // 4, 12, head_dim=256) == A and append(top // 4 + 1, 12, head_dim=256) == S

    def attend(rows, batch, heads, kv, weight):
        c = _cache(batch=batch, kv_heads=kv, table_width=rows // 16)
        return L.sherry_cache_attend_workspace(c, _attend(heads=heads, weight=FAKE if weight else None, row_stride=rows))
    assert attend(1024, 65535, 256, 256, False) > 0 and attend(1024, 65535, 257, 257, False) == 0
    assert attend(512, 65535, 257, 257, False) > 0 and attend(512, 65535, 257, 257, True) == 0
    assert attend(1024, 65535, 128, 128, True) > 0 and attend(1024, 65535, 129, 129, True) == 0
    assert attend(8192, 4096, 455, 455, True) > 0 and attend(8192, 4096, 456, 456, True) == 0

    def evict(batch, kv, keep, rows=64, **kw):
        c = _cache(batch=batch, kv_heads=kv, table_width=rows // 16)
        return L.sherry_cache_evict(c, _evict(keep=keep, out_stride=1 << 30, row_stride=1 << 30, kept=FAKE + 1, **kw), None)
    assert evict(1023, 4096, 1) == A and evict(1024, 4096, 1) == S
    assert evict(65535, 64, 1) == A and evict(65535, 65, 1) == S
    none = dict(weight_out=None, position_out=None)
    # rows of 64 bf16 values: 128 kept rows a workgroup; with room for all rows nothing moves
    assert evict(4096, 4, 1023 * 128, 1 << 20, **none) == A and evict(4096, 4, 1023 * 128 + 1, 1 << 20, **none) == S
    assert evict(4096, 4, 1024 * 128, 1 << 20, **none) == S and evict(4096, 4, 1024 * 128, 1024 * 128, **none) == A
    assert evict(4096, 4, 1023 * 1024) == A and evict(4096, 4, 1024 * 1024) == S
