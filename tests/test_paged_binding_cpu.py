"""What the Python side of the paged-cache calls refuses before anything reaches the library."""
import pytest
import torch

from paper_2511_12201_amd import binding as ob


@pytest.fixture
def call():
    """Q, K, pool, descriptor and counts of a call that only lacks a GPU."""
    dt = torch.bfloat16
    Q, K = torch.zeros(2, 4, 5, 64, dtype=dt), torch.zeros(2, 2, 5, 64, dtype=dt)
    pages, table = torch.zeros(8, 16, 64, dtype=dt), torch.zeros(2, 2, 2, dtype=torch.int32)
    pool = ob.make_page_pool(pages, pages.clone(), table)
    return (Q, K, pool, ob.make_chunk_desc(Q, K), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32),
            torch.zeros(2, 2, 32, dtype=torch.int32))


def test_a_turned_chunk_needs_its_queries(call):
    Q, K, pool, desc, cnt, ends, rows = call
    with pytest.raises(ValueError, match="Q"):
        ob.omni_paged_append(desc, ob.make_rope_desc(64), None, K, K, pool, cnt, cnt, ends, rows)


def test_a_pool_has_to_know_its_tensors(call):
    Q, K, pool, desc, cnt, ends, rows = call
    bare = ob.PagePool()
    bare.K, bare.V, bare.page_table = pool.K, pool.V, pool.page_table
    bare.n_pages, bare.page_rows, bare.pages_cap = pool.n_pages, pool.page_rows, pool.pages_cap
    for run in (lambda: ob.omni_paged_attn(desc, Q, bare, ends, cnt),
                lambda: ob.omni_paged_append(desc, None, None, K, K, bare, cnt, cnt, ends, rows),
                lambda: ob.omni_paged_evict(bare, 4, 0, 0, cnt, ends, rows, rows.float())):
        with pytest.raises(ValueError, match="make_page_pool"):
            run()


def test_scratch_on_another_device_is_refused(call):
    Q, K, pool, desc, cnt, ends, rows = call
    far = ob.Workspace("meta")
    for run in (lambda: ob.omni_paged_attn(desc, Q, pool, ends, cnt, ws=far),
                lambda: ob.omni_paged_evict(pool, 4, 0, 0, cnt, ends, rows, rows.float(), ws=far)):
        with pytest.raises(ValueError, match="workspace"):
            run()
