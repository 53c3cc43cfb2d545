"""Score candidate assignments with costs measured on this card.

    python examples/measured_costs.py [--bits 4] [--weights4] [--candidates 64] [--window 4096 --sinks 4]

Runs one layer of a served model (paged cache, position rotation, attention) on the GPU at a grid of lengths, puts the measured
times in the place of the roofline's attention term, and scores the same candidates with the roofline's cost tables and with the
measured ones.  With --weights4 the projections, the feed-forward block and the output head are held in 4 bits and measured too, and
the roofline beside them is that of the model in 4 bits.  The model is an 8B-class one (32 layers, 32 heads on 8), the trace the
small synthetic one; the weights and rows are random, which no time here depends on.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_07144_amd import binding, measured, traces  # noqa: E402

MODEL = np.array((32, 4096, 14336, 128256, 32, 8, 16), dtype=binding.MODEL_DTYPE)
GPU = np.array((288e9, 2.5e15, 8e12, 128e9, 1.075e12, 50e9, 8), dtype=binding.GPU_DTYPE)


def score(tr, tables, n):
    """Records of the trace's first n candidates with the given cost tables."""
    w = binding.ap_workload_create(tr.arrival_us, tr.prompt_len, tr.out_len)
    try:
        M = len(tr.t_on_us)
        binding.ap_costtable_set(w, np.zeros(M, np.uint32), tr.t_on_us, tr.t_off_us, tr.B, tr.slo_ttft_us, tr.slo_tpot_us, tr.penalty_us, *tables)
        rows = torch.from_numpy(tr.assignment_rows(0, n).view(np.int16)).cuda()
        out = torch.zeros((n, 8), dtype=torch.int64, device="cuda")
        binding.ap_eval_candidates(w, rows.data_ptr(), n, out.data_ptr(), torch.cuda.current_stream().cuda_stream)
        return out.cpu().numpy().view(binding.METRICS_DTYPE).reshape(-1)
    finally:
        binding.ap_workload_destroy(w)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--bits", type=int, choices=(16, 4), default=16, help="what the cache is held in")
    p.add_argument("--window", type=int, default=0, help="sliding window of the attention (0: none)")
    p.add_argument("--sinks", type=int, default=0, help="first tokens that stay visible beside the window")
    p.add_argument("--weights4", action="store_true", help="weights in 4 bits, measured too")
    p.add_argument("--candidates", type=int, default=64)
    a = p.parse_args(argv)
    model = MODEL.copy()
    if a.weights4:
        model["weight_bits"] = 4
    tr = traces.make_trace(0)
    longest = int((tr.prompt_len + tr.out_len).max())
    grid = np.unique(np.concatenate([2 ** np.arange(4, int(np.log2(longest)) + 1), [longest]]))
    decode_us, prefill_us = measured.layer_times(model, tr.B, grid, grid, bits=a.bits, window=a.window, sinks=a.sinks)
    print(f"one layer, {tr.B} slots, cache in {a.bits} bits: microseconds of append and attention")
    for n, d, f in zip(grid, decode_us, prefill_us):
        print(f"  {n:6d} tokens   decode step {d:9.1f}   prefill {f:9.1f}")
    w = binding.ap_workload_create(tr.arrival_us, tr.prompt_len, tr.out_len)
    roofline = binding.ap_roofline_costs(w, len(tr.prompt_len), np.array([model]), np.array([GPU]), np.array([(0, 0, 1, tr.B)], binding.GROUP_DTYPE))
    binding.ap_workload_destroy(w)
    weights = measured.weight_times(model, tr.B, grid) if a.weights4 else None
    if weights:
        print(f"one layer's weights in 4 bits: decode step {weights[0]:.1f} us, prefill of {grid[-1]} tokens {weights[1][-1]:.1f}; output head {weights[2]:.1f}")
    tables = measured.request_tables(model, GPU, tr.B, tr.prompt_len, tr.out_len, grid, decode_us, grid, prefill_us, weights)
    print(f"the roofline's model has weights in {model['weight_bits']} bits")
    for name, t in (("roofline", roofline), ("measured", tables)):
        m = score(tr, t[:2], a.candidates)
        print(f"{name}: mean TTFT {m['sum_ttft_us'].mean() / len(tr.prompt_len) / 1e3:8.2f} ms, mean TPOT {m['sum_tpot_us'].mean() / len(tr.prompt_len) / 1e3:7.3f} ms, "
              f"best p99 of E2E {m['p99_e2e_us'].min() / 1e3:9.1f} ms, best share within the SLO {m['slo_ok'].max() / len(tr.prompt_len):.3f}")
    return 0


if __name__ == "__main__":
    sys.exit(main())
