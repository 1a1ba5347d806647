"""The workspace of chunk_attn: its split goes by the device's compute units."""
import ctypes

import numpy as np

from paper_2608_23599_amd import binding as B


def test_split_goes_by_compute_units():
    """One row over a long exact context: at most three rounds of two workgroups a compute unit, each of
    which leaves 16 rows of 132 floats (a machine without a device counts as one unit)."""
    import torch
    cus = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 1
    cap = 1 << 15
    levels, lens, news = np.full((1, 1, cap), 16, np.int8), np.array([64 * cap]), np.array([1], np.int32)
    c = B.CacheStruct()
    c.B = c.Hkv = c.Hq = 1
    c.D, c.T, c.nblk_cap = 128, 64 * cap, cap
    c.level = c.koff = c.voff = c.arena = c.seq_len = 4096
    c.arena_bytes = 16384
    c.level_host, c.seq_len_host = levels.ctypes.data, lens.ctypes.data
    nb = int(B._chunk_ws(ctypes.byref(c), news.ctypes.data))
    assert 0 < nb <= 3 * 2 * cus * 16 * 132 * 4 + 256
