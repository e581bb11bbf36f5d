"""What the calls on 8-bit caches, pages and 4-bit weights refuse before anything reaches a GPU.  CPU only: the
addresses given here are never followed."""
import pytest

from paper_2504_11816_b200 import binding as B

A = 1 << 20        # an aligned address


def _refused(code, text, fn, *a, **kw):
    with pytest.raises(B.IsvError) as ei:
        fn(*a, **kw)
    assert ei.value.code == code and text in ei.value.message, ei.value


def test_q8_sizes():
    assert B.isv_q8_sizes(8, 128) == (8 * (32 * 128 + 16), 8 * 2 * 16 * 128 * 2)
    assert B.isv_q8_sizes(1, 80) == (32 * 80 + 16, 2 * 16 * 80 * 2)
    for heads, d in ((0, 64), (1, 96), (1, 0)):
        _refused(B.ISV_EINVAL, "head_dim", B.isv_q8_sizes, heads, d)


@pytest.mark.parametrize("kw,text", [
    (dict(q_heads=6), "multiple"), (dict(q_heads=0), "multiple"), (dict(kv_heads=0), "multiple"), (dict(head_dim=96), "head_dim"),
    (dict(dtype=2), "dtype"), (dict(format=2), "format"), (dict(max_seqs=0), "max_seqs"), (dict(max_seqs=4097), "max_seqs"),
    (dict(max_ctas=-1), "max_ctas"), (dict(q_heads=1 << 18), "query heads")])
def test_q8_create(kw, text):
    d = dict(q_heads=8, kv_heads=4, head_dim=64, dtype=0, format=0, max_seqs=4, max_ctas=0)
    d.update(kw)
    _refused(B.ISV_EINVAL, text, B.isv_q8_create, **d)


def test_q8_calls_need_a_handle():
    _refused(B.ISV_EINVAL, "null handle", B.isv_q8_attn, None, A, 1, A, A, 1, 1, A, A, A, None, 1)
    _refused(B.ISV_EINVAL, "null handle", B.isv_q8_write, None, A, 1, A, A, 1, 1, A, None, A, A, 64, 64, 1, 1)
    _refused(B.ISV_EINVAL, "null", B.isv_q8_status, None)
    _refused(B.ISV_EINVAL, "null handle", B.isv_q8_free, None)


def _copy(**kw):
    d = dict(dst_pool=A, n_dst_pages=4, src_pool=2 * A, n_src_pages=4, page_bytes=64, layers=1, dst_layer_stride=0,
             src_layer_stride=0, src_ids=3 * A, dst_ids=None, n=2)
    d.update(kw)
    return B.isv_pages_copy, d


@pytest.mark.parametrize("kw,text", [
    (dict(dst_pool=None), "required"), (dict(src_pool=None), "required"), (dict(src_ids=None), "required"),
    (dict(dst_pool=A + 8), "multiples of 16"), (dict(page_bytes=24), "multiples of 16"), (dict(page_bytes=0), "bad page size"),
    (dict(layers=0), "layers"), (dict(n=-1), "n ("), (dict(n_dst_pages=0), "page counts"), (dict(n_src_pages=0), "page counts"),
    (dict(layers=2, dst_layer_stride=240, src_layer_stride=256), "layer stride"),
    (dict(layers=2, dst_layer_stride=256, src_layer_stride=240), "layer stride"), (dict(src_layer_stride=8), "multiples of 16"),
    (dict(page_bytes=1 << 33, n=1 << 20), "too large"), (dict(page_bytes=1 << 34), "bad page size")])
def test_copy(kw, text):
    fn, d = _copy(**kw)
    _refused(B.ISV_EINVAL, text, fn, **d)


def test_copy_of_nothing_is_fine():
    fn, d = _copy(n=0)
    fn(**d)


def _table(fn, **kw):
    d = dict(block_table=A, lens=2 * A, n_rows=4, table_stride=8, max_blocks_per_seq=8, open_in_pool=1, n_pages=100)
    if fn is B.isv_pages_fork:
        d.update(parent=3 * A, table_out=4 * A, lens_out=5 * A, n_rows_out=4, copy_src=6 * A, copy_dst=7 * A)
    elif fn is B.isv_pages_resize:
        d.update(new_lens=3 * A)
    else:
        d.update(table_out=4 * A, src_ids=5 * A, dst_ids=6 * A, max_moves=50, counts=7 * A)
    d.update(kw)
    return d


@pytest.mark.parametrize("fn", [B.isv_pages_fork, B.isv_pages_resize, B.isv_pages_compact])
@pytest.mark.parametrize("kw,code,text", [
    (dict(block_table=None), B.ISV_EINVAL, "required"), (dict(lens=None), B.ISV_EINVAL, "required"),
    (dict(n_rows=-1), B.ISV_EINVAL, "rows"), (dict(n_rows=4097), B.ISV_EINVAL, "rows"), (dict(table_stride=7), B.ISV_EINVAL, "table row"),
    (dict(max_blocks_per_seq=0), B.ISV_EINVAL, "table row"), (dict(open_in_pool=2), B.ISV_EINVAL, "open_in_pool"),
    (dict(n_pages=0), B.ISV_EINVAL, "page count"), (dict(n_pages=B.ISV_PAGES_MAX + 1), B.ISV_ECAPACITY, "at most")])
def test_table_operations(fn, kw, code, text):
    _refused(code, text, fn, **_table(fn, **kw))


def test_table_operations_own_arguments():
    fork, resize, compact = B.isv_pages_fork, B.isv_pages_resize, B.isv_pages_compact
    for name in ("parent", "table_out", "lens_out", "copy_src", "copy_dst"):
        _refused(B.ISV_EINVAL, "required", fork, **_table(fork, **{name: None}))
    _refused(B.ISV_EINVAL, "rows", fork, **_table(fork, n_rows_out=5000))
    _refused(B.ISV_EINVAL, "overlap", fork, **_table(fork, table_out=A))
    _refused(B.ISV_EINVAL, "overlap", fork, **_table(fork, lens_out=2 * A + 12))
    _refused(B.ISV_EINVAL, "overlap", fork, **_table(fork, copy_dst=6 * A + 4))
    _refused(B.ISV_EINVAL, "required", resize, **_table(resize, new_lens=None))
    _refused(B.ISV_EINVAL, "overlap", resize, **_table(resize, new_lens=A + 16))
    for name in ("table_out", "src_ids", "dst_ids", "counts"):
        _refused(B.ISV_EINVAL, "required", compact, **_table(compact, **{name: None}))
    _refused(B.ISV_EINVAL, "max_moves", compact, **_table(compact, max_moves=49))
    _refused(B.ISV_EINVAL, "overlap", compact, **_table(compact, table_out=A + 4))
    _refused(B.ISV_EINVAL, "overlap", compact, **_table(compact, dst_ids=5 * A + 4))


@pytest.mark.parametrize("kw,text", [
    (dict(w4=None), "required"), (dict(scales=None), "required"), (dict(group=16), "group"), (dict(K=96), "multiple of the group"),
    (dict(K=0), "multiple of the group"), (dict(N=0), "bad N"), (dict(max_M=0), "max_M"), (dict(max_M=65), "max_M"),
    (dict(dtype=3), "dtype"), (dict(scales=A + 1), "aligned")])
def test_linear4_create(kw, text):
    d = dict(w4=A, scales=2 * A, N=16, K=128, group=64, dtype=0, max_M=4)
    d.update(kw)
    _refused(B.ISV_EINVAL, text, B.isv_linear4_create, **d)


def test_linear4_calls_need_a_handle():
    _refused(B.ISV_EINVAL, "null handle", B.isv_linear4_forward, None, A, A, None, 1)
    _refused(B.ISV_EINVAL, "null", B.isv_linear4_status, None)
    _refused(B.ISV_EINVAL, "null handle", B.isv_linear4_free, None)
