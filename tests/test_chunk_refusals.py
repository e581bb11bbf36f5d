"""What the calls on chunks of new tokens refuse before anything reaches a GPU.  CPU only: the addresses given here are
never followed."""
import math

import pytest

from paper_2504_11816_b200 import binding as B

A = 1 << 20        # an aligned address


def _refused(code, text, fn, *a, **kw):
    with pytest.raises(B.IsvError) as ei:
        fn(*a, **kw)
    assert ei.value.code == code and text in ei.value.message, ei.value


@pytest.mark.parametrize("kw,text", [
    (dict(q_heads=6), "multiple"), (dict(q_heads=0), "multiple"), (dict(kv_heads=0), "multiple"), (dict(head_dim=96), "head_dim"),
    (dict(dtype=2), "dtype"), (dict(max_seqs=0), "max_seqs"), (dict(max_seqs=4097), "max_seqs"), (dict(max_ctas=-1), "max_ctas"),
    (dict(q_heads=1 << 18), "query heads"), (dict(rotary_dim=-16), "rotary_dim"), (dict(rotary_dim=20), "rotary_dim"),
    (dict(rotary_dim=80), "rotary_dim"), (dict(rotary_pairs=2), "rotary_pairs"), (dict(rotary_axes=0), "rotary_axes"),
    (dict(rotary_axes=5), "rotary_axes"), (dict(scale=math.inf), "scale"), (dict(softcap=-1.0), "softcap"), (dict(softcap=math.nan), "softcap")])
def test_create(kw, text):
    d = dict(q_heads=8, kv_heads=4, head_dim=64, dtype=0, max_seqs=4, max_ctas=0)
    d.update(kw)
    _refused(B.ISV_EINVAL, text, B.isv_chunk_create, **d)


def test_calls_need_a_handle():
    _refused(B.ISV_EINVAL, "null handle", B.isv_chunk_attn, None, A, 1, A, 1, 1, A, None, None, 1, A, 64, None, None, 0, A, None, 1, 1)
    _refused(B.ISV_EINVAL, "null handle", B.isv_chunk_write, None, A, 1, A, 1, 1, A, None, None, 1, A, A, 64, A, 64, None, A, None, None, 1.0, 1, 1)
    _refused(B.ISV_EINVAL, "null", B.isv_chunk_status, None)
    _refused(B.ISV_EINVAL, "null handle", B.isv_chunk_free, None)


def _verify(**kw):
    d = dict(target=A, row_starts=None, n_rows=10, draft=2 * A, vocab=100, dtype=B.ISV_F32, drafted=3 * A, n_draft=4 * A, uniforms=5 * A,
             seq_lens=6 * A, n_seqs=2, max_draft=4, tokens=7 * A, accepted=8 * A, lens_out=9 * A)
    d.update(kw)
    return d


@pytest.mark.parametrize("kw,text", [
    (dict(target=None), "required"), (dict(drafted=None), "required"), (dict(n_draft=None), "required"), (dict(uniforms=None), "required"),
    (dict(tokens=None), "required"), (dict(accepted=None), "required"), (dict(seq_lens=None), "lens_out"), (dict(dtype=3), "dtype"),
    (dict(target=A + 2), "aligned"), (dict(draft=A + 1, dtype=B.ISV_F16), "aligned"), (dict(vocab=0), "vocab"), (dict(max_draft=0), "max_draft"),
    (dict(max_draft=1025), "max_draft"), (dict(n_seqs=-1), "n_seqs"), (dict(n_rows=-1), "n_rows"), (dict(n_rows=9), "n_rows")])
def test_verify(kw, text):
    _refused(B.ISV_EINVAL, text, B.isv_draft_verify, **_verify(**kw))


def test_verifying_nothing_is_fine():
    B.isv_draft_verify(**_verify(n_seqs=0, n_rows=0))
