"""Calibration of the tag -> bitwidth map (Sec. 3.1.3): distortions D_k(2), D_k(4) and token counts N_k of every tag from captured
queries, keys and values, as tkv_allocate_bits_greedy / _exhaustive take them.

For one layer's capture: tkv_quantize_rows puts the tokens of ONE tag at ONE width (all others stay unquantised), tkv_prefill_attention
replays the requests, tkv_head_distortion compares with the replay of unquantised rows.  Aggregated over heads by the largest, over
requests by the mean, over layers by the sum.  Quantiser, attention and distortions run in the library's kernels; this file keeps buffers, selects
tokens, and aggregates."""
from __future__ import annotations

import numpy as np
import torch

from . import harness, tkv


class Replay:
    """Buffers and plan for the replays of a set of packed requests (every layer has the same lengths)."""

    def __init__(self, seq_indptr, n_q_heads: int, n_kv_heads: int, sm_scale: float, device, key_axis: int = tkv.TKV_KEYS_PER_TOKEN):
        self.seq_indptr = np.ascontiguousarray(seq_indptr, np.int32)
        self.batch, self.n_tokens = self.seq_indptr.size - 1, int(self.seq_indptr[-1])
        self.d_indptr = torch.from_numpy(self.seq_indptr).to(device)
        self.sm_scale, self.device, self.key_axis = float(sm_scale), self.d_indptr.device, key_axis
        self.desc = tkv.tkv_desc.make(n_kv_heads, 0, 0, int2_key_axis=key_axis)
        self.plan = tkv.tkv_plan_prefill(self.desc, n_q_heads, self.seq_indptr, None, harness.default_shared_units(self.device))
        self.prefill = tkv.tkv_prefill.make(self.plan, self.device)
        rows, heads = (self.n_tokens, n_kv_heads, tkv.HEAD_DIM), (self.n_tokens, n_q_heads, tkv.HEAD_DIM)
        self.K, self.V = (torch.empty(rows, dtype=torch.float16, device=self.device) for _ in range(2))
        self.plain, self.out = (torch.empty(heads, dtype=torch.float16, device=self.device) for _ in range(2))
        self.by_head = torch.empty((self.batch, n_q_heads), dtype=torch.float64, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        size = max(16, tkv.tkv_prefill_workspace_bytes(self.desc, self.plan.n_slots, self.plan.tile_rows))
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        size = max(16, tkv.tkv_distortion_workspace_bytes(self.batch, self.n_tokens, n_q_heads))
        self.sums = torch.empty(size, dtype=torch.uint8, device=self.device)

    def widths(self, tags, tag: int, bits: int) -> np.ndarray:
        """u8[n_tokens]: `bits` for the tag's tokens, 0 for the others; with per-channel keys the last INT2 tokens of a request that
        fill no block of 32 are at INT4 (Sec. 3.2.1)."""
        out = np.where(np.asarray(tags) == tag, bits, 0).astype(np.uint8)
        if bits == 2 and self.key_axis == tkv.TKV_KEYS_PER_CHANNEL:
            for a, b in zip(self.seq_indptr[:-1], self.seq_indptr[1:]):
                at = a + np.flatnonzero(out[a:b] == 2)
                out[at[at.size - at.size % tkv.GROUP_SIZE:]] = 4
        return out

    def attention(self, q, K, V, widths, out):
        """Replays attention with rows at `widths` (host u8[n_tokens]), on the current stream of the replay's device."""
        if any(t.device != self.device for t in (q, K, V)):
            raise ValueError("q, K and V are on %s" % self.device)
        blocks = None
        if self.key_axis == tkv.TKV_KEYS_PER_CHANNEL:
            blocks = torch.from_numpy(tkv.tkv_plan_row_blocks(widths, self.seq_indptr)).to(self.device)
        bits = torch.from_numpy(widths).to(self.device)
        with torch.cuda.device(self.device):
            tkv.tkv_quantize_rows(self.desc, K, V, bits, blocks, self.K, self.V, self.status)
            tkv.tkv_prefill_attention(self.desc, q, self.K, self.V, None, None, self.prefill, self.sm_scale, out, self.workspace, self.status)

    def distortion(self, q, K, V, tags, tag: int, bits: int) -> torch.Tensor:
        """f64 [requests, heads] (valid until the next call); `attention` with no token quantised has filled `plain`."""
        self.attention(q, K, V, self.widths(tags, tag, bits), self.out)
        with torch.cuda.device(self.device):
            tkv.tkv_head_distortion(self.plain, self.out, self.d_indptr, self.by_head, self.sums)
        return self.by_head


def token_counts(tags, seq_indptr) -> np.ndarray:
    """N_k i64[56] over requests: the median for the instruction prefix (cached once for all), the sum for other tags."""
    per = np.stack([tkv.tkv_tag_counts(tags[a:b]) for a, b in zip(seq_indptr[:-1], seq_indptr[1:])]) if len(seq_indptr) > 1 else np.zeros((1, tkv.N_TAGS), np.int64)
    inst = np.arange(tkv.N_TAGS) % 7 == 0
    return np.where(inst, np.median(per, 0).astype(np.int64), per.sum(0))


def tag_distortions(layers, tags, seq_indptr, sm_scale: float, key_axis: int = tkv.TKV_KEYS_PER_TOKEN):
    """(N i64[56], D2 f64[56], D4 f64[56]).  layers: (q [T,Hq,128], K, V [T,Hkv,128]) device bf16 tensors of each captured layer (layers may
    lie on different devices), requests packed as seq_indptr (host i32[requests+1]) says; tags: host u8[T]."""
    tags = np.ascontiguousarray(tags, np.uint8)
    D = np.zeros((2, tkv.N_TAGS))
    replays = {}
    for q, K, V in layers:
        if q.device not in replays:
            replays[q.device] = Replay(seq_indptr, int(q.shape[1]), int(K.shape[1]), sm_scale, q.device, key_axis)
        replay = replays[q.device]
        replay.attention(q, K, V, np.zeros(tags.size, np.uint8), replay.plain)
        for tag in np.unique(tags):
            for row, bits in enumerate((2, 4)):
                D[row, tag] += float(replay.distortion(q, K, V, tags, int(tag), bits).amax(1).mean())
    for replay in replays.values():
        if int(replay.status.item()):
            raise RuntimeError("replay raised status %d" % int(replay.status.item()))
    return token_counts(tags, np.asarray(seq_indptr)), D[0], D[1]
