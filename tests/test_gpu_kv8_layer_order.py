"""A decode step as the README shows it: each layer writes its new row and attends over it before the next layer, and the
tables and lengths follow at the step's end, with merges."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import check_attention, i32, key_like, tables, to_bf16, to_pool8

pytestmark = pytest.mark.gpu


def test_each_layer_attends_to_the_steps_own_entry():
    m, d = umim(), dev()
    r = W.rng(90)
    B, layers, Hq, Hkv, D, P, steps = 5, 3, 8, 2, 128, 21, 20
    bt, n = tables(r, [0] * B + [P], columns=4, spare=B * (steps + 2))
    own, pre = bt[:B], bt[B:]
    free = [p for p in range(n) if p not in set(bt.ravel().tolist())]
    codes, scales = oracle.kv8.quantise(key_like(r, (layers, n, 2, Hkv, 16, D)))
    cache, status = to_pool8(m, codes, scales, d), m.new_status(d)
    lens = np.zeros(B, np.int32)
    block_table, seq_lens, prompt_table, prompt_lens = i32(own, d), i32(lens, d), i32(pre, d), i32([P], d)
    rows = torch.arange(B, device=d)
    ws = m.workspace(m.umim_decode_attention_shared_workspace_size(B, 1, Hq, Hkv, D), d)
    for step in range(steps):
        nk, nv, sk, sv = key_like(r, (4, B, layers, Hkv, D))
        fresh = np.array([free.pop() if x % 16 == 0 else -1 for x in lens], np.int32)
        merge_k = np.minimum(np.where(r.random(B) < 0.2, 2, 0), lens + 1)
        new_k, new_v, new_pages = to_bf16(nk, d), to_bf16(nv, d), i32(fresh, d)

        q = key_like(r, (layers, B, Hq, D))
        at = (seq_lens // 16).long()
        block_table[rows, at] = torch.where(seq_lens % 16 == 0, new_pages, block_table[rows, at])
        attended = seq_lens + 1
        out = []
        for layer in range(layers):
            m.umim_kv8_write(cache, layer, block_table, seq_lens, new_k[:, layer], new_v[:, layer], dev_status=status)
            out.append(m.umim_decode_attention_shared_kv8(to_bf16(q[layer], d), cache, layer, prompt_table, prompt_lens,
                                                          block_table, attended, workspace_buf=ws, dev_status=status))
        released = m.umim_kv8_append_merge(cache, block_table, seq_lens, new_k, new_v, new_pages, i32(merge_k, d), i32(range(B), d),
                                           to_bf16(sk, d), to_bf16(sv, d), dev_status=status)

        # the step's entries appended, attention over them, and only then the merges
        appended = oracle.kv8.append_merge(codes, scales, own, lens, nk, nv, fresh, [0] * B, [0] * B, sk, sv)
        values, powers = oracle.kv8.pool_values(*appended[:2]), oracle.kv8.scales(appended[1])
        for layer in range(layers):
            check_attention(out[layer], *oracle.kv8.attend(
                q[layer], values, layer, [[pre[0], t] for t in appended[2]], [[P, x] for x in lens + 1], row_scales=powers))
        codes, scales, own, lens, freed, rejected = oracle.kv8.append_merge(codes, scales, own, lens, nk, nv, fresh, merge_k,
                                                                            np.arange(B), sk, sv)
        assert rejected == [] and int(status.item()) == 0
        np.testing.assert_array_equal(block_table.cpu().numpy(), own)
        np.testing.assert_array_equal(seq_lens.cpu().numpy(), lens)
        np.testing.assert_array_equal(released.cpu().numpy(), freed)
        free += [p for p in freed.tolist() if p >= 0]
