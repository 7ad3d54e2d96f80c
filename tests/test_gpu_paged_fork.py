"""rest_pages_fork where a parent's length and its pages do not fit together."""
import numpy as np
import pytest

import paper_2311_08252_b200 as rest
from gpu_util import to_dev

pytestmark = pytest.mark.gpu


def test_a_length_without_its_pages_is_not_forked():
    """Context 0 gave all its pages back and kept its length, context 1 has fewer pages than its length asks
    for, context 2 a length below 0, context 3 nothing at all, context 4 is whole."""
    page, B, W, P = 16, 10, 4, 12
    refs, table = np.zeros(P, np.int32), np.full((B, W), -1, np.int32)
    n_pages, kv_len = np.zeros(B, np.int32), np.zeros(B, np.int32)
    kv_len[:5] = 40, 33, -1, 0, 20
    n_pages[1:5] = 2, 1, 0, 2
    table[1, :2], table[2, 0], table[4, :2] = (0, 1), 2, (3, 4)
    refs[:5] = 1
    dev = [to_dev(x) for x in (refs, table, n_pages, kv_len)]
    got = rest.rest_pages_fork(*dev, to_dev(np.arange(5, dtype=np.int32)), to_dev(np.arange(5, 10, dtype=np.int32)), page)
    src, dst, status = (t.tolist() for t in got)
    assert status == [rest.REST_CTX_BAD_PAGES] * 3 + [rest.REST_CTX_OK] * 2
    assert src == [-1, -1, -1, -1, 4] and dst == [-1, -1, -1, -1, 5]
    refs[3], refs[5] = 2, 1
    table[9, :2] = 3, 5
    n_pages[9], kv_len[9] = 2, 20
    for t, want in zip(dev, (refs, table, n_pages, kv_len)):
        assert np.array_equal(t.cpu().numpy(), want)


def test_without_the_context_that_does_not_fit_the_others_are_served():
    """Pages are counted out in order, a refused context's too; asked again without it, the later ones get theirs."""
    page, B, W, P = 16, 4, 6, 8
    dev = [to_dev(np.zeros(P, np.int32)), to_dev(np.full((B, W), -1, np.int32)), to_dev(np.zeros(B, np.int32))]
    need = np.array([3 * page, 6 * page, page, 0], np.int32)
    status = rest.rest_pages_reserve(*dev, to_dev(need), page).tolist()
    assert status == [rest.REST_CTX_OK, rest.REST_CTX_NO_PAGES, rest.REST_CTX_NO_PAGES, rest.REST_CTX_OK]
    need[1] = 0
    assert rest.rest_pages_reserve(*dev, to_dev(need), page).tolist() == [rest.REST_CTX_OK] * 4
    assert dev[2].tolist() == [3, 0, 1, 0] and dev[1][2, 0] == 3 and dev[0].tolist() == [1] * 4 + [0] * 4
