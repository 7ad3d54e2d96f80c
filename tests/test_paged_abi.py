"""What the paged-cache entry points refuse, checked on the host before anything is launched (the
pointers below are never dereferenced)."""
import ctypes

import numpy as np
import pytest

import paged_util as plain
import paper_2311_08252_b200 as rest

OK, INVALID, UNSUPPORTED = 0, 1, 2


def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


GOOD = strides(8 * 16 * 128, 16 * 128, 128)


def write(k=256, s=GOOD, P=4, page=16, table=256, ts=3, cols=3, new=strides(4096, 1024, 128), B=1, H_kv=8, N=4, D=128):
    return rest.lib().rest_paged_kv_write(k, 256, s, P, page, table, ts, cols, 256, 256, 256, new, None, B, H_kv, N, D,
                                          None)


def test_row_writes_refuse():
    assert write(B=0) == OK and write(N=0) == OK
    assert write(k=None) == INVALID and write(k=264) == INVALID          # null, not 16-byte aligned
    assert write(page=24) == UNSUPPORTED and write(page=8) == UNSUPPORTED and write(page=512) == UNSUPPORTED
    assert write(D=96) == UNSUPPORTED
    assert write(s=strides(16384, 2048, 124)) == INVALID                 # a row that starts off a 16-byte boundary
    assert write(s=strides(0, 2048, 128)) == INVALID                     # pages on top of one another
    assert write(table=None) == INVALID and write(ts=2) == INVALID and write(P=0) == INVALID
    assert write(new=strides(4096, 1024, 4)) == INVALID


def test_row_commits_refuse():
    c = lambda depth=4, B=1, page=16, nodes=256: rest.lib().rest_paged_kv_commit(  # noqa: E731
        256, 256, GOOD, 4, page, 256, 3, 3, 256, nodes, 256, B, 8, 64, 128, depth, None, None)
    assert c(B=0) == OK
    assert c(depth=17) == UNSUPPORTED and c(depth=0) == INVALID and c(page=20) == UNSUPPORTED and c(nodes=None) == INVALID


def test_page_calls_refuse():
    L = rest.lib()
    fork = lambda F=2, page=16, P=8, cols=4, ts=4: L.rest_pages_fork(  # noqa: E731
        256, P, 256, ts, cols, 256, 256, 4, page, 256, 256, F, 256, 256, 256, None)
    assert fork(F=0) == OK
    assert fork(F=1025) == UNSUPPORTED and fork(page=17) == UNSUPPORTED and fork(P=(1 << 20) + 1) == UNSUPPORTED
    assert fork(F=-1) == INVALID and fork(ts=3) == INVALID and fork(cols=0) == INVALID
    reserve = lambda B=2, page=16, P=8: L.rest_pages_reserve(  # noqa: E731
        256, P, 256, 4, 4, 256, 256, B, page, 256, None)
    assert reserve(B=0) == OK
    assert reserve(B=8193) == UNSUPPORTED and reserve(P=0) == INVALID and reserve(page=1) == UNSUPPORTED
    release = lambda window=0, sinks=0, page=16: L.rest_pages_release(  # noqa: E731
        256, 8, 256, 4, 4, 256, 256, 2, page, window, sinks, None)
    assert release(window=-1) == INVALID and release(sinks=-1) == INVALID and release(page=0) == UNSUPPORTED
    copy = lambda n=1, D=128, src=256: L.rest_pages_copy(256, 256, GOOD, 4, 16, 8, D, src, 256, n, None)  # noqa: E731
    assert copy(n=0) == OK
    assert copy(n=-1) == INVALID and copy(D=32) == UNSUPPORTED and copy(src=None) == INVALID


def test_python_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    t = torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(rest.RestError):
        rest.rest_pages_copy(t, t, i, i)
    with pytest.raises(rest.RestError):
        rest.rest_pages_reserve(i, i[None], i[:1], i[:1], 16)


def test_the_plain_model_shares_and_returns_pages():
    """The model itself: two forks of a context share its whole pages; everything released, all counts are 0."""
    page = 4
    refs, table = np.zeros(10, np.int32), np.full((3, 4), -1, np.int32)
    n_pages, kv_len = np.zeros(3, np.int32), np.zeros(3, np.int32)
    assert plain.reserve(refs, table, n_pages, np.array([10, 0, 0]), page).tolist() == [0, 0, 0]
    kv_len[0] = 10
    src, dst, st = plain.fork(refs, table, n_pages, kv_len, np.array([0, 0]), np.array([1, 2]), page)
    assert st.tolist() == [0, 0] and src.tolist() == [2, 2] and dst.tolist() == [3, 4]
    assert refs[:5].tolist() == [3, 3, 1, 1, 1] and kv_len.tolist() == [10] * 3
    plain.release(refs, table, n_pages, np.zeros(3, int), page)
    assert refs.sum() == 0 and (table == -1).all()


def attend(st=None, dtype=0, P=4, page=16, ts=3, cols=3, H=8, H_kv=2, N=4, D=128, window=0, sinks=0, scale=1.0, q=256,
           mask=256, B=1):
    st = strides(4096, 1024, 128, 4096, 2048, 128, 4096, 1024, 128) if st is None else st
    return rest.lib().rest_paged_attention(q, 256, 256, st, dtype, P, page, 256, ts, cols, 256, None, mask, B, H, H_kv,
                                           N, D, window, sinks, scale, 256, None, None, 0, None)


def test_attention_refuses():
    assert attend(B=0) == OK
    assert attend(D=96) == UNSUPPORTED and attend(N=257) == UNSUPPORTED and attend(H_kv=3) == UNSUPPORTED
    assert attend(page=8) == UNSUPPORTED and attend(page=48) == UNSUPPORTED
    assert attend(dtype=2) == INVALID and attend(dtype=-1) == INVALID
    assert attend(scale=0.0) == INVALID and attend(scale=float("inf")) == INVALID and attend(scale=float("nan")) == INVALID
    assert attend(window=-1) == INVALID and attend(sinks=-1) == INVALID and attend(P=0) == INVALID
    assert attend(q=None) == INVALID and attend(q=264) == INVALID and attend(ts=2) == INVALID
    assert attend(strides(4096, 1024, 128, 4096, 2048, 124, 4096, 1024, 128)) == INVALID
    assert attend(strides(4096, 1024, 128, 4096, 2048, 64, 4096, 1024, 128)) == INVALID      # rows that overlap
    assert rest.paged_attention_workspace_bytes(1, 8, 3, 4, 128) == 0
    assert rest.paged_attention_workspace_bytes(1, 8, 2, 4, 96) == 0


def sampled(dtype=0, V=100, B=1, N=4, depth=4, logits=256, ctx=500):
    return rest.lib().rest_accept_sampled(logits, dtype, ctx, 100, V, 256, 256, 256, 256, 256, 256, B, N, depth, 256, 256,
                                          256, None, 0, None)


def test_sampled_acceptance_refuses():
    assert sampled(B=0) == OK
    assert sampled(V=(1 << 18) + 1) == UNSUPPORTED and sampled(N=257) == UNSUPPORTED and sampled(depth=17) == UNSUPPORTED
    assert sampled(dtype=3) == INVALID and sampled(V=0) == INVALID and sampled(depth=0) == INVALID
    assert sampled(logits=257) == INVALID and sampled(logits=None) == INVALID and sampled(ctx=-1) == INVALID and sampled(B=-1) == INVALID
