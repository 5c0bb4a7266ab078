"""Masks and tables of angles without a value have no address, and would be taken for none at all
(a chain of drafts, heads as they are): the 16-bit cache's calls refuse them before they look
at anything on a device."""
import pytest
import torch


def batch():
    import paper_2503_21135_amd as pkg
    from paper_2503_21135_amd._lib import CacheDesc
    desc = CacheDesc()
    desc.n_pages, desc.n_heads, desc.head_dim, desc.page_size, desc.type = 8, 2, 64, 64, 0
    return pkg, desc, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.tensor([0, 2, 5]).int()


@pytest.mark.parametrize("shape", [(5, 0), (0,), ()])
def test_masks(shape):
    pkg, desc, table, lens, off = batch()
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    mask = torch.zeros(shape, dtype=torch.int64)
    with pytest.raises(pkg.MoEError, match="mask"):
        pkg.moe_tree_attention(desc, table, lens, off, 3, 23, q, q.clone(), 0.1, mask=mask)


@pytest.mark.parametrize("shape", [(0, 32), (50, 0), (0, 0), (32,)])
def test_tables_of_angles(shape):
    pkg, desc, table, lens, off = batch()
    q, k = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    tab = torch.zeros(shape)
    with pytest.raises(pkg.MoEError, match="cos"):
        pkg.moe_cache_append(desc, table, lens, off, 3, q, k, k, q.clone(), cos=tab, sin=tab)


@pytest.mark.gpu
def test_a_cache_on_the_device():
    import paper_2503_21135_amd as pkg
    cache, off = pkg.PagedCache.create(2, 64, 2, 64), torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    kv, q = (torch.randn(5, h, 64, device="cuda").to(torch.bfloat16) for h in (2, 4))
    cache.k.zero_(), cache.v.zero_()
    with pytest.raises(pkg.MoEError, match="mask"):
        cache.attend(q, off, 3, 23, mask=torch.zeros(5, 0, dtype=torch.int64, device="cuda"))
    for shape in ((0, 32), (50, 0), (32,)):
        none = torch.zeros(*shape, device="cuda")
        with pytest.raises(pkg.MoEError, match="cos"):
            cache.append(q, kv, kv, off, 3, cos=none, sin=none)
    assert not cache.k.any() and not cache.v.any()
    cache.append(q, kv, kv, off, 3)      # without a table, and without a mask: as they are, a chain
    out = cache.attend(q, off, 3, 23)
    ones = torch.tensor([[1], [3], [1], [3], [7]], dtype=torch.int64, device="cuda")
    assert torch.equal(cache.attend(q, off, 3, 23, mask=ones), out)
    none = cache.attend(q[:0], torch.zeros_like(off), 3, 23, mask=ones[:0])      # no tokens is fine
    assert none.shape == (0, 4, 64)
