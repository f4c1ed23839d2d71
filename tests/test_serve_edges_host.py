"""Host-side checks of the serving-layer operators: what the binding hands to the library (CPU only)."""
import ctypes as C
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


def test_windows_without_the_causal_mask_keep_their_splits(lib):
    """Without the mask a row sees up to the last key, as far behind its window as there are new tokens: a chunk's keys are split over
    workgroups (and need the workspace) as they are without the window; with the mask the window ends what a tile of rows sees."""
    P = 0x10000                                 # an address that no call here may reach
    c = vitq.vq_kv_cache(P, P, vitq.VQ_BF16, 1, 64, 16, 10000, 16 * 64, 16 * 64, 64, 1.0, 1.0)
    n = C.c_size_t()
    assert lib.vq_attention_paged_workspace(2000, 1, 1, C.byref(c), 2000, C.byref(n)) == 0 and n.value > 0
    name = lambda causal, window: vitq.STATUS_NAMES[lib.vq_attention_paged(
        P, vitq.VQ_BF16, 2000, 64, 1, P, P, 1, P, 4096, 4096, C.byref(c), 0.1, causal, window, 2000, P, 64, None, None, 0, None)]
    assert name(1, 0) == name(0, 0) == name(0, 100) == "VQ_ERR_WORKSPACE"
