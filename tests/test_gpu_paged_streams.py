"""Streams named by their handles."""
import pytest
import torch

import paper_2311_08252_b200 as rest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("handle", [0, 1, 2])                   # default, cudaStreamLegacy, cudaStreamPerThread
def test_the_default_streams_by_handle(handle):
    gen = torch.Generator("cuda").manual_seed(3)
    q, k, v = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((2, 3, 4, 64), (6, 2, 16, 64), (6, 2, 16, 64)))
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    kv_len = torch.tensor([30, 7], dtype=torch.int32, device="cuda")
    want = rest.rest_paged_attention(q, k, v, table, kv_len, None, 0.1)
    torch.cuda.synchronize()
    got = rest.rest_paged_attention(q, k, v, table, kv_len, None, 0.1, stream=handle)
    refs, n_pages = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    room = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    status = rest.rest_pages_reserve(refs, room, n_pages, kv_len, 16, stream=handle)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and status.tolist() == [0, 0] and room.tolist() == [[0, 1, -1], [2, -1, -1]]
