"""The three paged-cache operators over blocks that are denoised: a block's rows are appended once and rewritten in every
iteration, its queries see the whole prefix and the whole block; then the next block follows."""
import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged as oracle
from test_gpu_paged import BF, DEV, F32, U, compare, f64, status_word

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block,Hq,Hkv,room", [(8, 4, 2, 0), (32, 4, 2, 0), (32, 8, 2, 900)])
def test_blocks_that_are_rewritten(dtype, block, Hq, Hkv, room):
    """32 x 4 rows per KV head take the tcgen05 kernel where the table has room (bf16)."""
    B, D, ps = 3, 64, 16
    prompt, blocks, iterations = [37, 0, 300], 3, 2
    width = -(-(max(prompt) + blocks * block) // ps)
    n_pages = B * width
    g = torch.Generator().manual_seed(block)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    table, free, count = torch.zeros(B, width + room, dtype=torch.int32, device=DEV), torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV), i32([n_pages])
    kv_len, n_new, st = i32([0] * B), i32(prompt), status_word()
    kc, vc = (torch.full((n_pages, Hkv, ps, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    max_rows = max(sum(prompt), B * block)
    qkv = torch.zeros(max_rows, Hq + 2 * Hkv, D, dtype=dtype, device=DEV)
    w = torch.ones(D, dtype=dtype, device=DEV)
    pages = ds.PageUpdatePlan(kv_len, n_new, table, free, count, ps, max_rows, kv_len_out=kv_len, free_cnt_out=count, status=st)
    write = ds.QkNormRopePlan(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pages.positions, ds.RopeTable(D, 1e4), w, w,
                              k_cache=kc, v_cache=vc, slot_map=pages.slot_map, n_rows=pages.row_start[B:], status=st)
    attend = ds.PagedAttnPlan(write.q_out, kc, vc, table, kv_len, 0.125, row_start=pages.row_start, max_q=block, causal=False, status=st,
                              lse=torch.zeros(max_rows, Hq, dtype=F32, device=DEV))
    frequencies = oracle.rope_frequencies(D, 1e4)
    held = [(np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))) for _ in range(B)]

    def rows(n, starts):
        """What the cache has to hold of the new rows: K normed and rotated, within rounding, and V."""
        for b in range(B):
            x, pos = f64(qkv)[starts[b]:starts[b + 1]], np.arange(n[b]) + len(held[b][0])
            want, size = oracle.norm_rope(x[:, Hq:Hq + Hkv], np.ones(D), 1e-6, pos, *frequencies, False)
            slots = pages.slot_map[starts[b]:starts[b + 1]].cpu()
            k, v = (f64(c.transpose(1, 2).reshape(-1, Hkv, D)[slots]) for c in (kc, vc))
            assert (np.abs(k - want) <= (2.0 ** -8 if dtype == BF else U) * np.abs(want) + 64 * U * size).all()
            assert np.array_equal(v, x[:, Hq + Hkv:])
            yield k, v
    pages.launch()
    qkv.copy_(torch.randn(qkv.shape, generator=g))
    write.launch()                                           # the prompt: cached, nothing attends yet
    starts = np.concatenate([[0], np.cumsum(prompt)])
    held = list(rows(prompt, starts))
    n_new.fill_(block)
    starts = np.arange(B + 1, dtype=np.int32) * block
    for _ in range(blocks):
        pages.launch()
        assert kv_len.tolist() == [len(h[0]) + block for h in held]
        for _ in range(iterations):
            qkv.copy_(torch.randn(qkv.shape, generator=g))
            write.launch()
            attend.launch()
            assert ds.ds_read_status(st) == 0
            now = [tuple(np.concatenate(p) for p in zip(old, new)) for old, new in zip(held, rows([block] * B, starts))]
            top = max(len(k) for k, _ in now)
            dk, dv = np.zeros((2, B, Hkv, top, D))
            for b, (k, v) in enumerate(now):
                dk[b, :, :len(k)], dv[b, :, :len(k)] = k.transpose(1, 0, 2), v.transpose(1, 0, 2)
            n = B * block
            ref = oracle.attn_paged(f64(write.q_out)[:n], dk, dv, np.arange(B)[:, None], [len(k) for k, _ in now], starts, 0.125, False)
            compare(attend.out[:n], attend.lse[:n], ref, dtype, D, top)
        held = now
