"""No-GPU checks of attention's C calls at the ends of what they take: empty sides and the largest sizes."""
import ctypes
import os

import pytest

ONE = 4096                       # (an address that nothing reads: every call below is refused, or has nothing to do)


@pytest.fixture(scope="module")
def hot():
    from paper_2604_04736_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_04736_amd import build
        build.build_libhot()
    return binding


def _desc(hot, batch=2, heads=4, kv=2, queries=10, keys=12, width=16, **more):
    d = hot.hot_attention_desc()
    pitch = lambda h, n: hot.hot_pitch(h * n * width, n * width, width)      # noqa: E731
    d.batch, d.heads, d.kv_heads, d.queries, d.keys, d.width, d.dtype, d.table_dtype, d.scale = batch, heads, kv, queries, keys, width, 1, 1, 0.25
    for name in ("q", "o", "grad_o", "grad_q"):
        setattr(d, name, pitch(heads, queries))
    for name in ("k", "v", "grad_k", "grad_v"):
        setattr(d, name, pitch(kv, keys))
    for k, v in more.items():
        setattr(d, k, v)
    return d


def test_groups_of_no_tokens(hot):
    """An empty tensor's address is null: it is asked for where there are tokens alone."""
    lib = hot.lib()

    def forward(d, query_groups, key_groups):
        room = lib.hot_attention_workspace_bytes(ctypes.byref(d), 0)
        return lib.hot_attention_forward(ctypes.byref(d), ONE, ONE, ONE, *(None,) * 6, query_groups, key_groups, ONE, None, None, ONE, room, None)
    assert forward(_desc(hot, groups=2, queries=0), None, ONE) == 0
    assert forward(_desc(hot, groups=2, queries=0, keys=0), None, None) == 0
    assert forward(_desc(hot, groups=2, batch=0, keys=0), ONE, None) == 0
    assert forward(_desc(hot, groups=2, queries=0), None, None) == hot.HOT_EINVAL
    assert forward(_desc(hot, groups=2, batch=0, keys=0), None, None) == hot.HOT_EINVAL
    assert forward(_desc(hot, groups=2), None, ONE) == hot.HOT_EINVAL
    assert forward(_desc(hot, groups=2), ONE, None) == hot.HOT_EINVAL
    assert forward(_desc(hot, groups=2, queries=0), None, ONE + 2) == hot.HOT_EINVAL


def test_the_most_tokens(hot):
    """2^31 - 128 of either, so that where the last tile ends is a 32-bit number too; one more is refused."""
    lib, most = hot.lib(), (1 << 31) - 128
    one = dict(batch=1, heads=1, kv=1, width=8)
    for which in (0, 1):
        for sizes in (dict(queries=most, keys=4), dict(queries=4, keys=most), dict(queries=most, keys=most)):
            assert lib.hot_attention_workspace_bytes(ctypes.byref(_desc(hot, **one, **sizes)), which) > 0, sizes
            more = {n: size + (size == most) for n, size in sizes.items()}
            assert lib.hot_attention_workspace_bytes(ctypes.byref(_desc(hot, **one, **more)), which) == hot.HOT_EINVAL, more
        # rows of all heads of all entries
        assert lib.hot_attention_workspace_bytes(ctypes.byref(_desc(hot, 2, 1, 1, 4, 1 << 30, 8)), which) == hot.HOT_EINVAL
        # the line that queries lie on
        table = dict(tables=1, buckets=4, codes=21)
        last = (1 << 31) - 1 - 10
        assert lib.hot_attention_workspace_bytes(ctypes.byref(_desc(hot, first_query=last, **table)), which) > 0
        assert lib.hot_attention_workspace_bytes(ctypes.byref(_desc(hot, first_query=last + 1, **table)), which) == hot.HOT_EINVAL
