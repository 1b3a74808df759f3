"""Arrays of a cache, its boxes and its pool that a program replaces (the table
and references of a compaction into other arrays, for one): the library sees the
new ones, and nothing that it cannot use."""
import pytest
import torch

wk = pytest.importorskip("paper_2609_38121_amd")


def make():
    c = wk.WushKVCache(2, 2, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=200, device="cpu", page_order="none", n_pages=5)
    return c, wk.WushKVBounds(c), wk.WushKVPool(c)


ARRAYS = [(0, n) for n in ("pages", "page_table", "win_k", "win_v", "seq_len", "quant_end", "commit")]
ARRAYS += [(1, "codes"), (1, "scales"), (2, "refs"), (2, "held"), (2, "low")]


@pytest.mark.parametrize("which,name", ARRAYS)
def test_replaced_arrays_are_the_ones_described(which, name):
    of = make()[which]
    old = getattr(of, name)
    assert getattr(of.desc, name) == old.data_ptr()
    new = old.clone()
    setattr(of, name, new)
    assert getattr(of, name) is new and getattr(of.desc, name) == new.data_ptr()
    bad = [new.to(torch.float64), new.flatten()[:-1], new.reshape(-1, 1, 1, 1, 1), new.to("meta"), None]
    if new.dim() > 1:
        bad.append(new.transpose(0, 1).contiguous().transpose(0, 1) if new.shape[0] > 1 else new[:, ::2])
    for x in bad:
        with pytest.raises(ValueError):
            setattr(of, name, x)
        assert getattr(of, name) is new and getattr(of.desc, name) == new.data_ptr()


def test_clones_have_arrays_of_their_own():
    c, _, _ = make()
    d = c.clone()
    d.page_table = torch.zeros_like(d.page_table)
    assert d.desc.page_table == d.page_table.data_ptr() != c.desc.page_table == c.page_table.data_ptr()


def test_a_selection_workspace_serves_every_length_and_count():
    c, _, _ = make()
    sizes = {wk.wushkv_select_workspace_bytes(c, 4, n, k) for n in (0, 100, 200, 1 << 30) for k in (0, 3, 1000)}
    assert len(sizes) == 1 and sizes.pop() >= 4 * c.batch * c.n_kv_heads * c.max_pages
