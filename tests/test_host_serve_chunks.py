"""What the launch plan takes a cache for, without a GPU: the workspace says how many rows a chunk has."""
import ctypes as C

import paper_2306_03078_amd.serve_binding as S
from test_host_serve import descriptor


def workspace(**sizes):
    d = descriptor(**{**dict(heads=8, kv_heads=1, head_dim=128, page=16, layers=1, max_fresh=16), **sizes})
    return S._lib().spqr_tree_attention_workspace_bytes(C.byref(d))


def test_a_pool_that_many_requests_share_counts_once():
    """64 requests of 128 rows over 2 MB, each with a table as wide as the pool: as one request over it; 64 requests over 128 MB: not."""
    one = workspace(requests=1, pages=256, max_pages=256)
    assert workspace(requests=64, pages=256, max_pages=256) == one
    assert workspace(requests=64, pages=64 * 256, max_pages=256) > 3 * one
    assert workspace(requests=64, pages=64 * 256, max_pages=8) == one       # tables that reach 4 MB of it


def test_sizes_at_their_ends():
    for requests in (1, 1024):
        for pages in (1, (1 << 31) // 16 - 1):
            for max_pages in (1, (1 << 31) - 1):
                for kv in (1, 64, 1024):
                    assert workspace(requests=requests, pages=pages, max_pages=max_pages, heads=1024, kv_heads=kv, head_dim=256, max_fresh=256) > 0
