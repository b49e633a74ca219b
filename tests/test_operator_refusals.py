"""Calls of the rotation and paged-cache entry points that are refused on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

INVALID, SHAPE, DTYPE, CAPACITY = 1, 2, 3, 4
A = 1 << 20          # an aligned address that nothing ever reads


@pytest.fixture(scope="module")
def mst():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2408_11746_b200 as m
    return m


def _status(mst, f, *args, **kw):
    with pytest.raises(mst.MstError) as e:
        f(*args, **kw)
    return e.value.status


def _rot(mst, D=64, rot=64, f=A, gq=A, gk=A, eps=1e-6):
    return mst.Rotation(D, rot, f, gq, gk, eps)


def _fwd(mst, rot=None, dtype=1, tokens=4, seq=4, positions=None, hq=2, hk=2, Q=A, K=A, ld=128, Qo=A, Ko=A, ldo=128):
    mst.mst_qk_norm_rotate_fwd(rot if rot is not None else _rot(mst), dtype, tokens, seq, positions, hq, hk, Q, K, ld, Qo, Ko, ldo, stream=0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), DTYPE), (dict(tokens=-1), INVALID), (dict(hq=-1), INVALID), (dict(seq=0), INVALID), (dict(Q=None), INVALID),
    (dict(Ko=None), INVALID), (dict(ld=120), SHAPE), (dict(ldo=100), SHAPE), (dict(ld=132), SHAPE), (dict(Q=A + 8), SHAPE),
    (dict(Ko=A + 2), SHAPE), (dict(tokens=1 << 32), SHAPE), (dict(positions=A + 1), SHAPE), (dict(hq=65536, ld=1 << 23, ldo=1 << 23), SHAPE)])
def test_forward(mst, kw, status):
    assert _status(mst, _fwd, mst, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(D=60), SHAPE), (dict(D=264), SHAPE), (dict(D=0), SHAPE), (dict(rot=8), SHAPE), (dict(rot=80), SHAPE), (dict(rot=-16), SHAPE),
    (dict(f=None), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(gq=A + 4), SHAPE), (dict(f=A + 2), SHAPE)])
def test_rotation(mst, kw, status):
    assert _status(mst, _fwd, mst, rot=_rot(mst, **kw)) == status
    assert _status(mst, mst.mst_qk_norm_rotate_bwd_workspace, _rot(mst, **kw), 4) == status


def test_forward_of_nothing(mst):
    _fwd(mst, tokens=0)
    _fwd(mst, hq=0, hk=0, Q=None, K=None, Qo=None, Ko=None)


def _bwd(mst, rot=None, dtype=1, tokens=4, hq=2, hk=2, Q=A, K=A, ld=128, dQo=A, dKo=A, lddo=128, dQ=A, dK=A, ldg=128, gq=A, gk=A, ws=A,
         ws_bytes=1 << 20):
    rot = rot if rot is not None else _rot(mst)
    mst._check(mst._lib.mst_qk_norm_rotate_bwd(rot, dtype, tokens, 4, None, hq, hk, Q, K, ld, dQo, dKo, lddo, dQ, dK, ldg, gq, gk, ws, ws_bytes,
                                               None), "mst_qk_norm_rotate_bwd")


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), DTYPE), (dict(Q=None), INVALID), (dict(dKo=None), INVALID), (dict(dQ=None), INVALID), (dict(ldg=64), SHAPE),
    (dict(lddo=129), SHAPE), (dict(dQ=A + 4), SHAPE), (dict(gq=A + 2), SHAPE), (dict(ws=A + 4), SHAPE), (dict(ws=None), CAPACITY),
    (dict(ws_bytes=100), CAPACITY)])
def test_gradients(mst, kw, status):
    assert _status(mst, _bwd, mst, **kw) == status


def test_weight_gradient_without_a_weight(mst):
    assert _status(mst, _bwd, mst, rot=_rot(mst, gk=None)) == INVALID
    assert mst.mst_qk_norm_rotate_bwd_workspace(_rot(mst, gq=None, gk=None), 100) == 0
    assert mst.mst_qk_norm_rotate_bwd_workspace(_rot(mst), 100) > 0


def _cache(mst, **kw):
    c = mst.PagedCache(torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16), torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16))
    c.K = c.V = A
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(mst, **kw):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    b = mst.PagedBatch(i(3), i(2), i(2, 4), 8, 4, 64)
    b.first = b.len = b.page_table = A
    for k, v in kw.items():
        setattr(b, k, v)
    return b


BAD_CACHE = [(dict(K=None), INVALID), (dict(V=None), INVALID), (dict(page_size=0), INVALID), (dict(num_pages=-1), INVALID),
             (dict(kv_heads=0), INVALID), (dict(token_stride=100), SHAPE), (dict(token_stride=56), SHAPE), (dict(head_stride=8), SHAPE),
             (dict(page_stride=-2048), SHAPE), (dict(page_stride=8), SHAPE), (dict(K=A + 8), SHAPE)]
BAD_BATCH = [(dict(batch=-1), INVALID), (dict(tokens=-1), INVALID), (dict(first=None), INVALID), (dict(len=None), INVALID),
             (dict(page_table=None), INVALID), (dict(max_new=-1), INVALID), (dict(table_stride=-1), INVALID), (dict(first=A + 2), SHAPE),
             (dict(page_table=A + 1), SHAPE), (dict(batch=65536), SHAPE)]


def _append(mst, cache=None, batch=None, rot=None, heads=2, Q=A, K=A, V=A, ld=128, Qo=A, ldq=128):
    mst.mst_paged_append(cache or _cache(mst), batch or _batch(mst), rot, heads, Q, K, V, ld, Qo, ldq, stream=0)


def _attend(mst, cache=None, batch=None, heads=2, stride=64, Q=A, ldq=128, Out=A, ldo=128, lse=A, ws=A, ws_bytes=1 << 30):
    mst._check(mst._lib.mst_paged_attention(cache or _cache(mst), batch or _batch(mst), heads, stride, Q, ldq, Out, ldo, lse, ws, ws_bytes, None),
               "mst_paged_attention")


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_caches(mst, kw, status):
    assert _status(mst, _append, mst, cache=_cache(mst, **kw)) == status
    assert _status(mst, _attend, mst, cache=_cache(mst, **kw)) == status
    assert _status(mst, mst.mst_paged_attention_workspace, _cache(mst, **kw), _batch(mst), 2, 64) == status


@pytest.mark.parametrize("kw,status", BAD_BATCH)
def test_batches(mst, kw, status):
    assert _status(mst, _append, mst, batch=_batch(mst, **kw)) == status
    assert _status(mst, _attend, mst, batch=_batch(mst, **kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(K=None), INVALID), (dict(V=None), INVALID), (dict(heads=-1), INVALID), (dict(Q=None), INVALID), (dict(Qo=None), INVALID),
    (dict(ld=64), SHAPE), (dict(ldq=100), SHAPE), (dict(V=A + 8), SHAPE), (dict(Qo=A + 4), SHAPE), (dict(heads=65536), SHAPE)])
def test_append(mst, kw, status):
    assert _status(mst, _append, mst, **kw) == status


def test_append_with_a_rotation_of_another_width(mst):
    assert _status(mst, _append, mst, rot=_rot(mst, D=128)) == SHAPE
    assert _status(mst, _append, mst, cache=_cache(mst, head_dim=60)) == SHAPE


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), INVALID), (dict(heads=3), SHAPE), (dict(stride=0), INVALID), (dict(Q=None), INVALID), (dict(Out=None), INVALID),
    (dict(ldq=64), SHAPE), (dict(ldo=132), SHAPE), (dict(Q=A + 2), SHAPE), (dict(lse=A + 2), SHAPE), (dict(ws=A + 8), SHAPE)])
def test_attention(mst, kw, status):
    assert _status(mst, _attend, mst, **kw) == status


def test_attention_head_dims_and_workspaces(mst):
    for d in (32, 72, 256):
        assert _status(mst, _attend, mst, cache=_cache(mst, head_dim=d, token_stride=512, head_stride=256, page_stride=8192), ldq=512,
                       ldo=512) == SHAPE
    long = _batch(mst, max_len=8192, table_stride=512)
    need = mst.mst_paged_attention_workspace(_cache(mst), long, 2, 1 << 30)
    assert need > 0
    assert _status(mst, _attend, mst, batch=long, stride=1 << 30, ws=None, ws_bytes=0) == CAPACITY
    assert _status(mst, _attend, mst, batch=long, stride=1 << 30, ws_bytes=need - 1) == CAPACITY
    # distance one divides every distance: the same as no stride at all
    assert mst.mst_paged_attention_workspace(_cache(mst), long, 2, 1) == need


@pytest.mark.parametrize("max_new,max_len,stride,splits", [
    (1, 3000, 1 << 30, 6),          # few rows: 4 lists of 47 units of 64 entries, eight of them at least to a range
    (800, 20000, 1 << 30, 5),       # tiles: 52 blocks, for one wave of 296 (few rows: 400 blocks, two ranges)
    (200, 900, 1 << 30, 2),         # few rows: 4 lists of 25 tiles, 90 thousand entries
    (800, 20000, 64, 5),            # tiles again: 1.0 million entries
    (800, 4000, 64, 2),             # few rows: 0.3 million
    (4096, 1 << 20, 1 << 30, 1)])   # tiles: a wave of blocks as it is
def test_forms_of_the_attention(mst, max_new, max_len, stride, splits):
    """Kernel and ranges follow from what is said of the sizes; the workspace tells how many ranges there may be (148 SMs)."""
    n = mst.mst_paged_attention_workspace(_cache(mst), _batch(mst, tokens=1000, max_new=max_new, max_len=max_len), 4, stride)
    assert n == (splits * 1000 * 4 * 66 * 4 if splits > 1 else 0)


def test_form_of_the_attention_with_very_many_strided_keys(mst):
    """A table with room for 2^18 strided keys of a row or more: few rows, two ranges of 400 blocks."""
    for table, splits in (((1 << 20) - 4, 5), (1 << 20, 2)):
        b = _batch(mst, tokens=1000, max_new=800, max_len=20000, table_stride=table)
        assert mst.mst_paged_attention_workspace(_cache(mst), b, 4, 64) == splits * 1000 * 4 * 66 * 4


def test_calls_without_sequences(mst):
    none = _batch(mst, batch=0, first=None, len=None, page_table=None)
    _append(mst, batch=none)
    _attend(mst, batch=none)
    _attend(mst, batch=_batch(mst, tokens=0))


def test_structures_check_their_tensors(mst):
    z = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    for K, V in ((z, z[:2]), (z.float(), z.float()), (z, z.transpose(1, 2).contiguous().transpose(1, 2)), (z[..., ::2], z[..., ::2]), (z[0], z[0])):
        with pytest.raises(ValueError):
            mst.PagedCache(K, V)
    t = z.transpose(1, 2).contiguous().transpose(1, 2)
    assert (mst.PagedCache(t, t).token_stride, mst.PagedCache(t, t).head_stride) == (64, 1024)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    for a in ((i(2), i(2), i(2, 4)), (i(3), i(2), i(3, 4)), (i(3).long(), i(2), i(2, 4)), (i(3), i(2), i(2, 8)[:, ::2]), (i(3), i(2), i(2))):
        with pytest.raises(ValueError):
            mst.PagedBatch(*a, 4, 1, 1)
    assert ctypes.sizeof(mst.PagedCache) == 56 and ctypes.sizeof(mst.PagedBatch) == 48 and ctypes.sizeof(mst.Rotation) == 40


def test_rotation_checks_its_tensors(mst):
    """The library reads rot_dim / 2 and head_dim floats at the addresses it is given: tensors that hold something else are refused."""
    w, f = torch.ones(64), torch.ones(32)
    for args in ((w, w, w), (f[:31], w, w), (f.double(), w, w), (f.view(2, 16), w, w), (w[::2], w, w), (f, w.bfloat16(), w), (f, w, w.half()),
                 (f, w[:63], w), (f, w, torch.ones(128)), (f, torch.ones(128)[::2], w), (f, w, torch.ones(2, 64)), (f.int(), None, None)):
        with pytest.raises(ValueError):
            mst.Rotation(64, 64, *args)
    for args in ((f, w, w), (f, None, w), (f, None, None), (A, A, A), (torch.ones(65)[1:33], torch.ones(128)[64:], w)):
        mst.Rotation(64, 64, *args)
    mst.Rotation(64, 0, None, w, w)
    mst.Rotation(64, 0, torch.empty(0), w, w)
    mst.Rotation(64, 0, f, None, None)


@pytest.mark.parametrize("kw", [
    dict(num_pages=1 << 10, page_stride=1 << 58), dict(num_pages=(1 << 10) + 1, page_stride=1 << 57), dict(num_pages=(1 << 31) - 1, page_stride=(1 << 63) - 8),
    dict(num_pages=2, page_stride=1 << 56), dict(page_size=1 << 30, token_stride=1 << 34, page_stride=1 << 40), dict(page_size=1 << 12, token_stride=1 << 55),
    dict(kv_heads=1 << 10, head_stride=1 << 58), dict(kv_heads=2, head_stride=1 << 56)])
def test_strides_beyond_any_address(mst, kw):
    """Products of strides and counts that do not fit 64 bits are not taken for small ones."""
    c = _cache(mst, **kw)
    heads = c.kv_heads
    assert _status(mst, _append, mst, cache=c, heads=heads, ld=heads * 64, ldq=heads * 64) == SHAPE
    assert _status(mst, _attend, mst, cache=c, heads=heads, ldq=heads * 64, ldo=heads * 64) == SHAPE
    assert _status(mst, mst.mst_paged_attention_workspace, c, _batch(mst), heads, 64) == SHAPE


@pytest.mark.parametrize("kw", [
    dict(token_stride=64, head_stride=64), dict(token_stride=64), dict(token_stride=120), dict(page_stride=64), dict(page_stride=2040),
    dict(token_stride=64, head_stride=16 * 64 - 8), dict(token_stride=64, head_stride=1024, page_stride=2040),
    dict(page_stride=64, token_stride=3 * 64 - 8, head_stride=16 * 192), dict(head_stride=56), dict(kv_heads=1, token_stride=56),
    dict(kv_heads=1, num_pages=1, token_stride=0), dict(page_size=1, kv_heads=1, page_stride=0)])
def test_caches_whose_rows_overlap(mst, kw):
    """An append to rows that overlap has no defined result."""
    c = _cache(mst, **kw)
    assert _status(mst, _append, mst, cache=c, heads=c.kv_heads) == SHAPE
    assert _status(mst, _attend, mst, cache=c, heads=c.kv_heads) == SHAPE
    assert _status(mst, mst.mst_paged_attention_workspace, c, _batch(mst), c.kv_heads, 64) == SHAPE


@pytest.mark.parametrize("kw", [
    dict(), dict(token_stride=64, head_stride=1024), dict(token_stride=136, head_stride=72, page_stride=4096), dict(page_stride=128, token_stride=384),
    dict(page_stride=16 * 64, token_stride=64, head_stride=3 * 16 * 64), dict(kv_heads=1, head_stride=0, token_stride=64), dict(num_pages=1, page_stride=0),
    dict(num_pages=0, page_stride=0), dict(page_size=1, token_stride=0, page_stride=128), dict(page_stride=4096)])
def test_orders_that_are_no_overlap(mst, kw):
    c = _cache(mst, **kw)
    none = _batch(mst, tokens=0)
    _append(mst, cache=c, batch=none, heads=c.kv_heads)
    _attend(mst, cache=c, batch=none, heads=c.kv_heads)


def test_append_of_keys_and_values_to_one_place(mst):
    assert _status(mst, _append, mst, cache=_cache(mst, K=A, V=A)) == INVALID
    _append(mst, cache=_cache(mst, K=A, V=A), batch=_batch(mst, tokens=0))


def test_rows_of_no_tokens_have_no_address(mst):
    """An empty tensor's address is NULL: a step without tokens is no wrong argument, as in the products."""
    none = _batch(mst, tokens=0)
    _fwd(mst, tokens=0, Q=None, K=None, Qo=None, Ko=None)
    _bwd(mst, tokens=0, Q=None, K=None, dQo=None, dKo=None, dQ=None, dK=None, gq=None, gk=None)
    _append(mst, batch=none, Q=None, K=None, V=None, Qo=None)
    _append(mst, batch=none, K=None, V=None)
    _attend(mst, batch=none, Q=None, Out=None, lse=None, ws=None, ws_bytes=0)
    q = torch.empty((0, 128), dtype=torch.bfloat16)
    mst.mst_paged_attention(_cache(mst), none, 2, 64, q, q.stride(0), q, q.stride(0), torch.empty((2, 0)), torch.empty(0), stream=0)
    for f, kw in ((_fwd, dict(tokens=0, ld=100, Q=None)), (_append, dict(batch=none, ld=100, K=None)), (_attend, dict(batch=none, ldq=100, Q=None))):
        assert _status(mst, f, mst, **kw) == SHAPE


def test_form_of_the_attention_with_very_many_pages(mst):
    """A table with room for 2^27 pages of a sequence or more: few rows."""
    for table, splits in (((1 << 27) - 1, 5), (1 << 27, 2), ((1 << 31) - 1, 2)):
        b = _batch(mst, tokens=1000, max_new=800, max_len=20000, table_stride=table)
        assert mst.mst_paged_attention_workspace(_cache(mst), b, 4, 1 << 30) == splits * 1000 * 4 * 66 * 4


def test_positions_check_their_type(mst):
    """arange's own type is int64: read as int32, every other position would be 0."""
    p = torch.arange(8)
    for bad in (p, p.float(), p.int()[::2], p.int().view(2, 4), p.int()[:3]):
        with pytest.raises(ValueError):
            _fwd(mst, tokens=4, positions=bad)
        with pytest.raises(ValueError):
            mst.mst_qk_norm_rotate_bwd(_rot(mst), 1, 4, 4, bad, 2, 2, A, A, 128, A, A, 128, A, A, 128, stream=0)
    _fwd(mst, tokens=0, positions=p.int()[:0])
    assert _status(mst, _fwd, mst, tokens=4, positions=p.int(), dtype=9) == DTYPE       # further checks are the library's


def test_positions_of_no_tokens_have_no_address(mst):
    none = torch.empty(0, dtype=torch.int32)
    _fwd(mst, tokens=0, seq=0, positions=none, Q=None, K=None, Qo=None, Ko=None)
    mst.mst_qk_norm_rotate_bwd(_rot(mst), 1, 0, 0, none, 2, 2, None, None, 128, None, None, 128, None, None, 128, stream=0)
