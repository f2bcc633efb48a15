"""What the operators around a shared cache refuse before they look for a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2511_07423_amd as s
from paper_2511_07423_amd import binding as b


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=63), dict(head_dim=64, rot_dim=66), dict(head_dim=64, rot_dim=31), dict(head_dim=64, rot_dim=0),
    dict(base=1.0), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")), dict(magnitude=float("nan")),
    dict(scaling=("linear", 0.0)), dict(scaling=("linear", -1.0)), dict(scaling=("linear", float("inf"))),
    dict(scaling=("bands", 8.0, 4.0, 4.0, 8192.0)), dict(scaling=("bands", 8.0, -1.0, 4.0, 8192.0)), dict(scaling=("bands", 8.0, 1.0, 4.0, 0.0)),
    dict(scaling=("bands", 0.0, 1.0, 4.0, 8192.0)), dict(inv_freq=np.full(32, np.nan))])
def test_rope_descriptions(bad):
    with pytest.raises(s.SyneraError) as e:
        s.Rope(**{**dict(head_dim=64), **bad})
    assert e.value.status == s.EINVAL


def test_rope_limits_and_words():
    with pytest.raises(s.SyneraError) as e:
        s.Rope(258)
    assert e.value.status == s.EUNSUP
    for bad in (dict(layout="other"), dict(scaling=("other", 1.0))):
        with pytest.raises(KeyError):
            s.Rope(64, **bad)
    for bad in (dict(scaling=("linear",)), dict(scaling=("bands", 1.0)), dict(inv_freq=np.ones(31))):
        with pytest.raises(ValueError):
            s.Rope(64, **bad)
    desc = b._RopeDesc(64, 64, 2, 0, 10000.0, 0, 0, 0, 0, 1.0, None)
    h = C.c_void_p(1)
    assert b._lib.synera_rope_create(C.byref(h), C.byref(desc)) == s.EINVAL and h.value is None
    desc.layout, desc.scaling = 0, 3
    assert b._lib.synera_rope_create(C.byref(h), C.byref(desc)) == s.EINVAL
    assert b._lib.synera_rope_create(C.byref(h), None) == s.EINVAL
    assert b._lib.synera_rope_create(None, C.byref(desc)) == s.EINVAL
    assert b._lib.synera_rope_destroy(None) == s.OK


@pytest.mark.parametrize("args,status", [((0, 1, 64, 1, 1, 1), s.EINVAL), ((4, 0, 64, 1, 1, 1), s.EINVAL), ((4, 4, 64, 0, 1, 1), s.EINVAL),
                                         ((4, 4, 64, 1, 0, 1), s.EINVAL), ((4, 4, 64, 1, 1, 0), s.EINVAL), ((4, 3, 64, 1, 1, 1), s.EUNSUP),
                                         ((4, 4, 96, 1, 1, 1), s.EUNSUP), ((2048, 8, 64, 1, 1, 1), s.EUNSUP),
                                         ((1024, 8, 64, 1, 1 << 20, 1), s.EUNSUP), ((4, 4, 64, 1 << 16, 1, 1 << 14), s.EUNSUP)])
def test_batch_limits(args, status):
    with pytest.raises(s.SyneraError) as e:
        s.SharedBatch(*args)
    assert e.value.status == status


def test_null_handles():
    lib, one = b._lib, b._pack_heads(16, 16, 0, 1, 64, 64, 64, 64)
    table, n = np.zeros((1, 1), np.int32), np.ones(1, np.int32)
    p = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))                                   # noqa: E731
    assert lib.synera_rope_apply(None, 0, 1, 16, one, None, None) == s.EINVAL
    assert lib.synera_qk_norm_rope(None, 0, 1, 16, one, None, 0.0, None) == s.EINVAL
    assert lib.synera_batch_plan(None, 1, p(n), p(n), p(table), 1, 1, None) == s.EINVAL
    assert lib.synera_append_rope(None, None, 0, one, one, one, 0.0, 16, 16, None) == s.EINVAL
    assert lib.synera_shared_attention(None, one, 16, 16, 0.0, None, None) == s.EINVAL
    assert lib.synera_batch_destroy(None) == s.OK
    assert lib.synera_batch_create(None, 4, 4, 64, 1, 1, 1) == s.EINVAL
    for args in ((1, None, p(n), p(table)), (1, p(n), None, p(table)), (1, p(n), p(n), None), (0, p(n), p(n), p(table))):
        assert lib.synera_validate_shared(*args, 1, 1, 1, 1) == s.EINVAL
    with pytest.raises(ValueError):
        s.validate_shared([1, 2], [1], table, 1, 1, 1)


def test_a_magnitude_has_to_be_finite_in_32_bits():
    for bad in (1e39, -1e300):
        with pytest.raises(s.SyneraError) as e:
            s.Rope(64, magnitude=bad)
        assert e.value.status == s.EINVAL


@pytest.mark.parametrize("bad", [
    dict(n_q_heads=1), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=-2), dict(n_kv_heads=0), dict(n_kv_heads=-2), dict(slots=0), dict(max_tokens=0),
    dict(max_tokens=2), dict(max_pages=0), dict(max_pages=1), dict(B=0), dict(which=-1), dict(which=9), dict(ctx=-1), dict(new=-1),
    dict(ctx=(1 << 31) - 100, max_pages=1 << 27)])
def test_the_planning_hook_refuses_what_it_cannot_plan(bad):
    """Head counts that do not divide, sizes below one, lengths beyond the table: no division by zero, no read past the table."""
    a = {**dict(n_q_heads=2, n_kv_heads=2, slots=4, max_tokens=3, B=1, ctx=15, new=3, max_pages=2, which=0), **bad}
    ctx, new, table = np.array([a["ctx"]], np.int32), np.array([a["new"]], np.int32), np.array([[0, 1]], np.int32)
    p = lambda v: v.ctypes.data_as(C.POINTER(C.c_int32))                                   # noqa: E731
    out, n = np.zeros(64, np.int32), C.c_int64(0)
    assert b._lib.synera_debug_shared_plan(a["n_q_heads"], a["n_kv_heads"], a["slots"], a["max_tokens"], a["B"], p(ctx), p(new), p(table),
                                           a["max_pages"], a["which"], p(out), 64, C.byref(n), None) == s.EINVAL


def test_the_planning_hook_from_python():
    for hq, hkv in ((1, 2), (3, 2), (2, 0)):
        with pytest.raises(s.SyneraError) as e:
            s.debug_shared_plan(hq, hkv, 4, [3], [1], [[0]])
        assert e.value.status == s.EINVAL
    assert s.debug_shared_plan(2, 2, 4, [3], [1], [[0]])["head"][0, 0] == 1


@pytest.mark.parametrize("bad", [dict(scaling=("linear", 5e-324)), dict(scaling=("bands", 5e-324, 1.0, 4.0, 8192.0)), dict(scaling=("linear", 1e-300)),
                                 dict(inv_freq=np.full(32, 1e308)), dict(inv_freq=np.r_[np.ones(31), -1e300])])
def test_frequencies_turn_by_finite_angles_at_every_position(bad):
    """pos f / 2 pi is formed in 64 bits for any int32 position: frequencies that are infinite there, or become so, are refused."""
    with pytest.raises(s.SyneraError) as e:
        s.Rope(64, **bad)
    assert e.value.status == s.EINVAL
