"""What the operators for trees and logits refuse before they look for a GPU."""
import ctypes as C

import pytest
import torch

import paper_2511_07423_amd as s
from paper_2511_07423_amd import binding as b


@pytest.mark.parametrize("args,status", [((0, 1, 64, 1, 1, 1), s.EINVAL), ((4, 0, 64, 1, 1, 1), s.EINVAL), ((4, 4, 64, 0, 1, 1), s.EINVAL),
                                         ((4, 4, 64, 1, 0, 1), s.EINVAL), ((4, 4, 64, 1, 1, 0), s.EINVAL), ((4, 3, 64, 1, 1, 1), s.EUNSUP),
                                         ((4, 4, 96, 1, 1, 1), s.EUNSUP), ((2048, 8, 64, 1, 1, 1), s.EUNSUP),
                                         ((1024, 8, 64, 1, 1 << 20, 1), s.EUNSUP), ((4, 4, 64, 1 << 16, 1, 1 << 14), s.EUNSUP)])
def test_tree_limits(args, status):
    with pytest.raises(s.SyneraError) as e:
        s.TreeBatch(*args)
    assert e.value.status == status


@pytest.mark.parametrize("max_batch", [(1 << 14) + 1, 1 << 16, 1 << 20, (1 << 20) + 1])
def test_tree_limit_of_requests(max_batch):
    """A plan's time grows as the square of the requests."""
    with pytest.raises(s.SyneraError) as e:
        s.TreeBatch(4, 4, 64, max_batch, 1 << 20, 1)
    assert e.value.status == s.EUNSUP


def test_null_handles():
    lib = b._lib
    one = b._pack_heads(16, 16, 0, 1, 64, 64, 64, 64)
    assert lib.synera_tree_create(None, 4, 4, 64, 1, 1, 1) == s.EINVAL
    assert lib.synera_tree_plan(None, 1, 16, 16, 16, 1, 16, 1, 1, None, None) == s.EINVAL
    assert lib.synera_tree_append_rope(None, None, 0, one, one, one, 0.0, 16, 16, None) == s.EINVAL
    assert lib.synera_tree_attention(None, one, 16, 16, 0.0, None, None) == s.EINVAL
    assert lib.synera_tree_accept(None, 1, 16, 16, 16, 16, 16, 16, 16, 16, None) == s.EINVAL
    assert lib.synera_tree_commit(None, 1, 16, 16, 1, 0, 16, 16, None) == s.EINVAL
    assert lib.synera_tree_destroy(None) == s.OK


def test_null_handle_of_a_plan_with_held_pages():
    assert b._lib.synera_tree_plan_held(None, 1, 16, 16, 16, 1, 16, 1, 16, 1, None, None) == s.EINVAL


def test_pages():
    good = [1, 64, 128, None, 192, 4, 256, 320, 384, 10, 5, 448, 512, 576, 640, None]
    for at, bad in ((0, 0), (0, -1), (1, None), (2, None), (4, None), (5, 0), (6, None), (7, None), (8, None), (9, 0), (10, -1), (11, None), (12, None),
                    (13, None), (14, None), (1, 66), (3, 67), (13, 577)):
        args = list(good)
        args[at] = bad
        assert b._lib.synera_pages_update(*args) == s.EINVAL, (at, bad)
    for at, bad in ((4, 500), (6, 128), (11, 64), (12, 380), (13, 64), (3, 384)):        # one on another
        args = list(good)
        args[at] = bad
        assert b._lib.synera_pages_update(*args) == s.EINVAL, (at, bad)
    for at, bad in ((9, 1 << 27), (5, 1 << 27)):
        args = list(good)
        args[at] = bad
        assert b._lib.synera_pages_update(*args) == s.EUNSUP, (at, bad)


def desc(**more):
    names = [n for n, _ in b._LogitsDesc._fields_]
    at = {n: 0 for n in names} | dict(B=2, dtype=0, rows=2, vocab=40, in_stride=40, out_stride=40) | more
    return b._pack_logits(*(at[n] for n in names))


def test_the_description_is_as_long_as_the_structure():
    assert len(desc()) == C.sizeof(b._LogitsDesc)


@pytest.mark.parametrize("bad,status", [
    (dict(B=-1), s.EINVAL), (dict(rows=-1), s.EINVAL), (dict(vocab=0), s.EINVAL), (dict(dtype=3), s.EINVAL), (dict(rows=3), s.EINVAL),
    (dict(in_stride=39), s.EINVAL), (dict(out_stride=39), s.EINVAL), (dict(d_history=64), s.EINVAL), (dict(d_bias_id=64), s.EINVAL),
    (dict(d_bias=64), s.EINVAL), (dict(d_tokens=64, d_cu=64), s.EINVAL), (dict(d_tokens=64, d_parent=64), s.EINVAL), (dict(d_mask=66), s.EINVAL),
    (dict(history_columns=-1), s.EINVAL), (dict(bias_columns=-1), s.EINVAL), (dict(vocab=(1 << 30) + 1), s.EUNSUP), (dict(bias_columns=1023), s.EUNSUP),
    (dict(history_columns=1 << 19), s.EUNSUP), (dict(B=65536, rows=65536), s.EUNSUP),
    (dict(d_cu=64, d_tokens=64, d_parent=64, rows=(1 << 19) + 1), s.EUNSUP)])
def test_logits(bad, status):
    assert b._lib.synera_logits_adjust(desc(**bad), 1 << 20, 1 << 21, None) == status


def test_logits_that_lie_on_others():
    call, at = b._lib.synera_logits_adjust, 1 << 20
    assert call(None, at, at, None) == s.EINVAL
    assert call(desc(), None, at, None) == s.EINVAL and call(desc(), at, None, None) == s.EINVAL
    assert call(desc(), at + 2, at + 4096, None) == s.EINVAL
    assert call(desc(), at, at + 160, None) == s.EINVAL                      # one row further
    assert call(desc(out_stride=80), at, at, None) == s.EINVAL               # in place, but for the stride
    assert call(desc(d_mask=at + 300), 1 << 22, at, None) == s.EINVAL         # the output on the masks
    assert call(desc(d_presence=at + 316), 1 << 22, at, None) == s.EINVAL
    assert call(desc(rows=0, B=0), None, None, None) == s.OK


def test_tensors_that_are_not_on_the_gpu():
    x = torch.zeros((2, 40))
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        s.adjust_logits(x)
    with pytest.raises(ValueError):
        s.update_pages(i[:, None], i, i, i[:1], i, i, 0)
