"""Host-side checks of the serving-layer operators: what the binding hands to the library (CPU only)."""
import os

import pytest
import torch

from paper_2504_18547_amd import vitq


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(vitq.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return vitq.lib()


def test_page_tables_whose_rows_overlap_are_refused(lib, monkeypatch):
    """Rows closer than their columns (one history expanded to several sequences): the library sees the stride as it is."""
    monkeypatch.setattr(vitq, "_here", lambda *t: None)
    monkeypatch.setattr(vitq, "_stream", lambda: None)
    cache = vitq.KvCache(*[torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)])
    q = torch.zeros(3, 4 * 64, dtype=torch.bfloat16)
    offsets, lens = torch.tensor([0, 1, 2, 3]).int(), torch.tensor([40, 40, 40]).int()
    row = torch.arange(4, dtype=torch.int32)
    for table in (row.view(1, 4).expand(3, 4), torch.arange(8, dtype=torch.int32).as_strided((3, 4), (2, 1)), row[:1].view(1, 1).expand(3, 1)):
        with pytest.raises(vitq.VitqError) as e:
            vitq.vq_attention_paged(q, offsets, lens, table, cache, 0.125, True, 0, 0, torch.empty_like(q), None, None)
        assert vitq.STATUS_NAMES[e.value.status] == "VQ_ERR_STRIDE"
