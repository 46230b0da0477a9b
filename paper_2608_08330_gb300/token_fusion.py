"""Token fusion of one frame: every BEV cell of the ego map attends to every cell
of every present agent's map (an example of the token-memory operators).

    python -m paper_2608_08330_gb300.token_fusion --workload tiny --absent 1

The frame runs through the library as usual.  Then each agent's feature slot
becomes tokens: rtcc_memory_append finds their rows (agent k's slot of the memory
is its map's H' x W' cells), rtcc_qkv_prepare norms and rotates queries and keys by
(t, y, x) = (agent, metres, metres) and writes keys, values and coordinates to the
memory, and rtcc_memory_attention lets the ego's cells attend to it, with capped
scores, a bias that falls with distance, and absent agents' slots hidden.  As in the
built-in attention fusion there are no learned projections: a cell's feature vector,
cut into heads, is its query, key and value.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

THETA, EPS, CAP = 10000.0, 1e-6, 30.0


def head_layout(channels: int):
    """(heads, channels per head): heads of 64, or 32 for narrow maps."""
    if channels < 32 or channels % 32:
        raise ValueError(f"{channels} channels are not heads of 64 or 32")
    dim = 64 if channels % 64 == 0 else 32
    return channels // dim, dim


def axis_pairs(dim: int):
    """Channel pairs turned by t (agent), y and x: a quarter, three and three eighths."""
    t = dim // 8
    return t, (dim // 2 - t) // 2, dim // 2 - t - (dim // 2 - t) // 2


def workspace_bytes(tokens: int, keys: int, heads: int, dim: int) -> int:
    """Room for a part per 65,536 keys, and one more, so that no float32 sum of the attention gets long."""
    return (-(-keys // 65536) + 1) * tokens * heads * (dim + 2) * 4


def slopes(heads: int) -> np.ndarray:
    """Distance slopes per head, 1/4 per metre down to 1/256."""
    return (0.25 * 2.0 ** (-6.0 * np.arange(heads) / max(heads, 1))).astype(np.float32)


def positions(agent: int, feat_h: int, feat_w: int, cell: float) -> np.ndarray:
    """(t, y, x) of an agent's cells, row by row; the maps share the ego's frame."""
    y, x = np.divmod(np.arange(feat_h * feat_w), feat_w)
    return np.stack([np.full(y.shape, agent), y * cell, x * cell], axis=1).astype(np.float32)


def fuse(maps, dtype: str, feat_h: int, feat_w: int, cell: float):
    """Fused ego map and its log-sum-exps.

    maps: per agent its feature slot as uint16 [H' * W' * C] (rtcc_get_tensor), None
    = absent; the ego (agent 0) is present.  Returns torch tensors on the device:
    out [H' * W', heads, dim] in the storage type and lse [H' * W', heads]."""
    import torch

    from . import rtcc as R
    if not maps or maps[0] is None:
        raise ValueError("the ego's map (agent 0) is needed")
    dev = torch.device("cuda")
    kind = torch.bfloat16 if dtype == "bf16" else torch.float16
    code = R.BF16 if dtype == "bf16" else R.FP16
    cells, agents = feat_h * feat_w, len(maps)
    heads, dim = head_layout(maps[0].size // cells)
    stream = torch.cuda.current_stream().cuda_stream
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    empty = lambda *s, t=torch.int32: torch.empty(*s, dtype=t, device=dev)  # noqa: E731

    here = [k for k in range(agents) if maps[k] is not None]
    feats = torch.from_numpy(np.concatenate([maps[k] for k in here]).view(np.int16)).to(dev).view(kind)
    feats = feats.reshape(len(here) * cells, heads, dim)
    pos = torch.from_numpy(np.concatenate([positions(k, feat_h, feat_w, cell) for k in here])).to(dev)
    tokens, rows_all = feats.shape[0], agents * cells

    # rows of the present agents' tokens: sequence k owns slot k
    fresh, held = i32([cells if m is not None else 0 for m in maps]), i32([0] * agents)
    offsets, rows, begin, end, length = empty(agents + 1), empty(tokens), empty(agents), empty(agents), empty(agents)
    R.check(R.rtcc_memory_append(agents, cells, tokens, fresh.data_ptr(), held.data_ptr(), None, offsets.data_ptr(),
                                 rows.data_ptr(), None, None, begin.data_ptr(), end.data_ptr(), length.data_ptr(),
                                 stream), "rtcc_memory_append")

    # queries of every token (the ego's are used), keys and values into the memory
    q, k_mem, v_mem = empty(tokens, heads, dim, t=kind), empty(rows_all, heads, dim, t=kind), empty(rows_all, heads, dim, t=kind)
    coord = empty(rows_all, 2, t=torch.float32)
    st = (heads * dim, dim)
    cfg = R.prepare_config(heads, heads, dim, code, tokens, rows_all, st, st, st, st, st, st, axis_pairs(dim), theta=THETA,
                           eps=EPS)
    f = feats.data_ptr()
    R.check(R.rtcc_qkv_prepare(cfg, f, f, f, None, None, pos.data_ptr(), rows.data_ptr(), q.data_ptr(), k_mem.data_ptr(),
                               v_mem.data_ptr(), coord.data_ptr(), stream), "rtcc_qkv_prepare")

    # the ego's cells over the whole memory
    out, lse = empty(cells, heads, dim, t=kind), empty(cells, heads, t=torch.float32)
    slope = torch.from_numpy(slopes(heads)).to(dev)
    present = i32([int(m is not None) for m in maps])
    q_offsets, first, last = i32([0, cells]), i32([0]), i32([rows_all])
    workspace = empty(workspace_bytes(cells, rows_all, heads, dim), t=torch.uint8)
    cfg = R.attn_config(heads, heads, dim, code, cells, rows_all, st, st, st, st, 1, cells, rows_all, n_slots=agents,
                        slot_rows=cells, q_pos_row=3, cap=CAP)
    R.check(R.rtcc_memory_attention(cfg, q.data_ptr(), k_mem.data_ptr(), v_mem.data_ptr(), q_offsets.data_ptr(),
                                    first.data_ptr(), last.data_ptr(), None, present.data_ptr(), slope.data_ptr(),
                                    pos[:, 1:].data_ptr(), coord.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                    workspace.data_ptr(), workspace.numel(), stream), "rtcc_memory_attention")
    R.check(R.rtcc_memory_attention_status(stream), "rtcc_memory_attention")
    return out, lse


def frame_maps(workload: str, frame: int, absent=()):
    """Feature slots of one frame of a synthetic workload, None where absent."""
    import synth

    from . import build as B
    from . import rtcc as R
    B.build()
    cfg = synth.get_config(workload)
    ctx = R.rtcc_init(R.model_config(cfg), synth.weight_blob(synth.weights_for(cfg)))
    try:
        R.check(R.rtcc_frame_begin(ctx, frame + 1, 0.0), "rtcc_frame_begin")
        for k in range(cfg.n_agents):
            if k in absent:
                R.check(R.rtcc_payload_absent(ctx, k, float(k)), "rtcc_payload_absent")
            else:
                R.check(R.rtcc_payload_complete(ctx, k, synth.points_for(cfg, frame, k), float(k)), "rtcc_payload_complete")
        s, _, _ = R.rtcc_wait_detection(ctx, 60000)
        R.check(s, "rtcc_wait_detection")
        maps = [None if k in absent else R.rtcc_get_tensor(ctx, k, R.TENSOR_FEAT) for k in range(cfg.n_agents)]
    finally:
        R.rtcc_destroy(ctx)
    return cfg, maps


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="pp3")
    ap.add_argument("--frame", type=int, default=0)
    ap.add_argument("--absent", type=int, nargs="*", default=[], help="agents that do not report (not the ego)")
    a = ap.parse_args(argv)
    import synth
    agents = synth.get_config(a.workload).n_agents
    if any(not 0 < k < agents for k in a.absent):
        ap.error(f"--absent takes agents 1 to {agents - 1}: agent 0 is the ego")
    cfg, maps = frame_maps(a.workload, a.frame, a.absent)
    out, lse = fuse(maps, cfg.dtype, cfg.feat_h, cfg.feat_w, cfg.pillar * cfg.feat_stride)
    print(f"{a.workload}: {cfg.feat_h} x {cfg.feat_w} cells over {sum(m is not None for m in maps)} maps, "
          f"{out.shape[1]} heads of {out.shape[2]}: mean |out| {out.float().abs().mean().item():.4f}, "
          f"lse {lse.min().item():.3f} .. {lse.max().item():.3f}")
    return 0


if __name__ == "__main__":
    sys.exit(main())
