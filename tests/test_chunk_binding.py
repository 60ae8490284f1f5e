"""What the binding of the chunk operators refuses before anything reaches the library (no GPU)."""
import ctypes
import os

import pytest
import torch

import paper_2609_29364_b200.api as api
from test_chunk_host import ROOT, _context


def _tables(**over):
    i32, i64 = torch.int32, torch.int64
    return {**dict(ctx_len=torch.zeros(2, dtype=i32), new_len=torch.zeros(2, dtype=i32), held=torch.zeros((2, 4), dtype=i32),
                   n_held=torch.zeros(2, dtype=i32), free_blocks=torch.zeros(3, dtype=i32), free_begin=None,
                   kv_indptr=torch.zeros(3, dtype=i64), kv_indices=torch.zeros(5, dtype=i32), q_indptr=torch.zeros(3, dtype=i64),
                   slot_map=torch.zeros(4, dtype=i64), positions=torch.zeros(4, dtype=i32), row_req=None,
                   n_held_new=torch.zeros(2, dtype=i32), free_end=torch.zeros(1, dtype=i64)), **over}


def test_row_outputs_of_no_elements_are_not_left_out_ones():
    for over in (dict(slot_map=torch.zeros(0, dtype=torch.int64)), dict(positions=torch.zeros(0, dtype=torch.int32)),
                 dict(slot_map=None, positions=torch.zeros(0, dtype=torch.int32), row_req=torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(ValueError, match="one length"):
            _context().nsd_block_tables(**_tables(**over))


def test_tensors_that_the_device_cannot_read_are_refused():
    """Right in type and shape, but in pageable memory: a kernel would fault on the address."""
    c, bf = _context(), torch.bfloat16
    with pytest.raises(ValueError, match="cuda:0"):
        c.nsd_block_tables(**_tables())
    q, k, out = torch.zeros((3, 512), dtype=bf), torch.zeros((3, 128), dtype=bf), torch.zeros((3, 8, 64), dtype=bf)
    pos, slots, pool = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros((1, 4, 2, 2, 16, 64), dtype=bf)
    with pytest.raises(ValueError, match="cuda:0"):
        c.nsd_rope_append(pool, 0, q, k, k, out, pos, [32], torch.ones(32), slots)
    plan, i = torch.zeros(256, dtype=torch.uint8), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="cuda:0"):
        c.nsd_chunk_plan(plan, 3, i, torch.zeros(1, dtype=torch.int32), i)
    with pytest.raises(ValueError, match="cuda:0"):
        c.nsd_chunk_attn(plan, 3, pool, q, out, None, torch.zeros(4, dtype=torch.int32))


def test_the_documented_limit_of_heads_is_a_context_s():
    """Up to 32 q heads per kv head: what a context with the smallest max_gamma allows."""
    words = " ".join(open(os.path.join(ROOT, "include", "nsd.h")).read().replace("*", " ").split())
    assert "at most 32 q heads" in words and "128 q heads" not in words
    lib = api.load_library()

    def workspace(heads):
        return lib.nsd_workspace_bytes(ctypes.byref(api.NsdConfig(
            num_layers=1, num_slabs=1, num_q_heads=heads, num_kv_heads=1, head_dim=64, block_size=16, num_blocks=4, max_batch=1,
            max_gamma=1, vocab_size=2, max_table_entries=4)))

    assert workspace(32) > 0 and workspace(33) == 0
