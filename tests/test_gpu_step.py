"""A captured decode step of agents that share a prompt: page tables, norm and rotation, append, attention over the shared
prompt and the sequences' own tokens, replayed across page ends without the host, against the oracle's cache."""
import math

import numpy as np
import pytest
import torch

import gpu_common as gc
from paper_2605_17170_amd import harness, tkv
from paper_2605_17170_amd import workloads as wl
from test_gpu_shared import check, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.mark.parametrize("key_axis", [0, 1])
def test_steps_of_a_captured_loop(key_axis):
    from oracle import tkv_oracle
    tkv_oracle.build()
    batch, hk, r, prompt, steps = 3, 2, 4, 333, 70
    hq, heads = hk * r, hk * r + 2 * hk
    n_seqs, max_pages = 1 + batch, 8
    desc = tkv.tkv_desc.make(hk, 12, 20, int2_key_axis=key_axis)
    pool = torch.full((tkv.tkv_pool_bytes(desc),), 0xFF, dtype=torch.uint8, device=DEV)
    bit_map, status = torch.zeros(32, dtype=torch.uint8, device=DEV), i32(1)
    table = tkv.tkv_table.make(i32(n_seqs, max_pages), i32(n_seqs), i32(n_seqs), i32(32), i32(2))
    tkv.tkv_table_reset(desc, table)
    rows, n2, n4 = table.tensors[:3]
    rope = tkv.tkv_rope_make(128, 1e6, [24, 20, 20], interleaved=True, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    weights = [(1.0 + 0.2 * torch.randn(128, device=DEV, generator=g)).to(torch.bfloat16) for _ in range(2)]

    def projection(tokens):
        return torch.randn((tokens, heads, 128), device=DEV, generator=g).to(torch.bfloat16)

    def step_of(tokens, lens, tags, offset):
        """The calls for `tokens` tokens that arrive in buffers of their own; (buffers, function)."""
        work = tkv.tkv_table_max_work(n_seqs, tokens)
        b = {"qkv": projection(tokens), "pos": i32(tokens), "pos3": i32(3, tokens), "wp": i32(work), "ws": i32(work, 64), "nw": i32(1),
             "q": torch.empty((tokens, hq, 128), dtype=torch.bfloat16, device=DEV), "k": torch.empty((tokens, hk, 128), dtype=torch.bfloat16, device=DEV),
             "v": torch.empty((tokens, hk, 128), dtype=torch.bfloat16, device=DEV), "lens": dev(np.array(lens, np.int32)), "tags": dev(np.array(tags, np.uint8)),
             "tmp": torch.empty(tkv.tkv_table_workspace_bytes(n_seqs, tokens), dtype=torch.uint8, device=DEV)}

        def call():
            tkv.tkv_table_append(desc, table, None, None, b["lens"], b["tags"], None, b["pos"], None, b["wp"], b["ws"], b["nw"], b["tmp"], status)
            b["pos3"].copy_((b["pos"] + offset)[None].expand(3, -1))
            parts = torch.split(b["qkv"], [hq, hk, hk], 1)
            tkv.tkv_norm_rope(rope, *parts, b["pos3"], *weights, 1e-6, b["q"], b["k"], b["v"])
            tkv.tkv_quantize_append(desc, pool, bit_map, b["k"], b["v"], b["tags"], b["wp"], b["ws"], status)
        return b, call

    # the prompt, then a first question of each agent
    rng = np.random.default_rng(3)
    tags = rng.choice([2, 4], prompt).astype(np.uint8)
    first = [20, 64, 3]
    own_tags = [rng.choice([2, 4], n).astype(np.uint8) for n in first]
    if key_axis:
        tags, own_tags = tkv.tkv_route_residual(tags), [tkv.tkv_route_residual(t) for t in own_tags]
    lists_k, lists_v, lists_bits = [[] for _ in range(n_seqs)], [[] for _ in range(n_seqs)], [[] for _ in range(n_seqs)]

    def record(b, lens, tags):
        k, v, at = b["k"].cpu().view(torch.int16).numpy().view(np.uint16), b["v"].cpu().view(torch.int16).numpy().view(np.uint16), 0
        for s, n in enumerate(lens):
            lists_k[s].append(k[at:at + n]); lists_v[s].append(v[at:at + n]); lists_bits[s].append(np.asarray(tags[at:at + n], np.uint8))
            at += n

    for lens, t, offset in (([prompt, 0, 0, 0], tags, 0), ([0] + first, np.concatenate(own_tags), prompt)):
        b, call = step_of(len(t), lens, t, offset)
        call()
        torch.cuda.synchronize()
        record(b, lens, t)

    # a plan for the pages that the sequences will have at the end; the tables grow into it
    have2, have4 = n2.cpu().numpy(), n4.cpu().numpy()
    grown = have4[1:] + steps
    counts = -(-have2[1:] // 64) + -(-grown // 64)
    items, sip = tkv.tkv_plan_decode(desc, np.concatenate([[0], np.cumsum(counts)]), have2[1:], grown, 12)
    plan = tkv.tkv_plan_decode_shared(desc, batch, hq, have2[:1], have4[:1], [0, batch], list(range(batch)), 2, items, sip)
    indptr = dev((np.arange(n_seqs + 1) * max_pages).astype(np.int32))
    prefix = tkv.tkv_prefix.make(indptr[:2], rows.view(-1), n2[:1], n4[:1], dev(np.array([0, batch], np.int32)), dev(np.arange(batch, dtype=np.int32)),
                                 dev(plan.member_slots), dev(plan.prefix_items), plan.max_members)
    out = torch.empty((batch, hq, 128), dtype=torch.bfloat16, device=DEV)
    workspace = torch.empty(tkv.tkv_decode_workspace_bytes(desc, plan.n_slots, hq), dtype=torch.uint8, device=DEV)
    d_items, d_slots = dev(plan.items), dev(plan.seq_item_indptr)
    b, write = step_of(batch, [0, 1, 1, 1], [4] * batch, prompt)

    def step():
        write()
        tkv.tkv_decode_attention_shared(desc, pool, bit_map, b["q"], indptr[1:], rows.view(-1), n2[1:], n4[1:], d_items, prefix, d_slots, plan.n_slots,
                                        1.0 / math.sqrt(128.0), out, workspace, status)

    step()
    torch.cuda.synchronize()
    record(b, [0, 1, 1, 1], [4] * batch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for s in range(1, steps):
        b["qkv"].copy_(projection(batch))
        graph.replay()
        torch.cuda.synchronize()
        record(b, [0, 1, 1, 1], [4] * batch)
        assert b["pos"].tolist() == [first[i] + s for i in range(batch)]
        if s not in (1, 2, 40, 43, 44, 45, 60, 61, 62, steps - 1):
            continue
        Ks, Vs = [], []
        for k, v, bits in zip(lists_k, lists_v, lists_bits):
            K, V, t = np.concatenate(k), np.concatenate(v), np.concatenate(bits)
            if key_axis:
                # blocks of INT2 keys arrive within one chunk, all in the first one here
                Kq, Vq = gc.orc.quantize(K, t), gc.orc.quantize(V, t)
                tok = gc.orc.int2_blocks(t, 0)
                scale, zero = gc.orc.quantize_k_channel(K, tok, Kq[0])
                Kh, Vh = gc.kc_dequantized(Kq, Vq, tok, scale, zero)
            else:
                Kh, Vh = gc.orc.dequantize(*gc.orc.quantize(K, t)), gc.orc.dequantize(*gc.orc.quantize(V, t))
            Ks.append(np.asarray(Kh, np.float64)); Vs.append(np.asarray(Vh, np.float64))
        q = b["q"].cpu().view(torch.int16).numpy().view(np.uint16)
        check(out, reference(q, Ks, Vs, [[0, 1, 2]], hk), "step %d" % s)
    assert int(status.item()) == 0
    assert n4.tolist() == [int(have4[0])] + (have4[1:] + steps).tolist() and n2.tolist() == have2.tolist()
