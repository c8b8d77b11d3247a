"""Compare the rollout engine with its KV cache in bf16 and in 4 bits, on the same weights and tokens.

For each set of sequences (how many, their contexts): the time of a decode step and of the prefill, the time of
decode attention and of its append per layer, and the KV pool.  Then, for the first layers of the model alone, how far the two
caches' logits and log-probabilities of given tokens are apart.  Typical use, from the repository root:

    python3 -u paper_2509_21009_amd/cache_compare.py --out profiles/kv4_engine.md

Weights are random (the workload's, seeded): a layer's attention averages values that have nothing to do with each other, so that
the quantiser's error does not average out against a common part as it does in a trained model, and each layer adds to it.  The
differences say what 4 bits do to these sums, not what a trained model loses by them.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

SETS = ((64, 600, 4500), (330, 128, 1280), (16, 2000, 14000), (1, 14000, 14000))


def _tokens(n, lo, hi, vocab):
    rng = np.random.default_rng(n)
    plens = rng.integers(lo, hi + 1, n)
    offs = np.concatenate([[0], np.cumsum(plens)])
    return plens, offs, rng.integers(0, vocab, offs[-1]).astype(np.int32)


def _engine(rp, shape, weights, plens, new, kv4):
    return rp.Engine(shape, weights, max_seqs=len(plens), max_prefill_tokens=16384, max_context=int(plens.max()) + new,
                     kv_pages=int(np.sum((plens + new + 63) // 64)) + 16, kv4=kv4)


def times(rp, eng, plens, toks, offs, new):
    """Least step and prefill ms of three rollouts, and us a launch of the kernel classes of one profiled rollout more."""
    ids, max_new, best = np.arange(len(plens)), np.full(len(plens), new, np.int32), (np.inf, np.inf)
    for _ in range(3):
        s = eng.rollout(ids, toks, offs, max_new, 7, 1.0)[1][0]
        best = np.minimum(best, (s["decode_ms"] / s["decode_steps"], s["makespan_ms"] - s["decode_ms"]))
    eng.profile(list(rp.KERNEL_CLASSES))
    eng.rollout(ids, toks, offs, max_new, 7, 1.0)
    us = {(p["phase"], p["kernel"]): 1e3 * p["total_ms"] / p["launches"] for p in eng.profile_read()}
    eng.profile([])
    return best[0], best[1], us


def logits(torch, eng, plens, toks, offs, forced):
    """Logits after each given token, [steps, rows, vocab] on the host."""
    n, steps = forced.shape
    eng.prefill(np.arange(n), toks, offs, np.full(n, steps + 1, np.int32))
    out = [eng.decode_step(forced_tokens=forced[:, j], logits=True)[2].float().cpu() for j in range(steps)]
    eng.abort(np.arange(n))
    return torch.stack(out)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="7b-long")
    ap.add_argument("--new", type=int, default=48, help="tokens decoded in the timed rollouts")
    ap.add_argument("--sets", default=None, help="n:lo:hi,... instead of the usual ones")
    ap.add_argument("--layers", default="1,2,4,8", help="depths at which logits are compared")
    ap.add_argument("--out", default=None, help="also write the tables there")
    args = ap.parse_args()

    import torch

    from paper_2509_21009_amd import rollpack as rp
    from workloads import make_weights, make_workload
    from workloads.gen import truncated

    rp.load_library()
    lines = []

    def put(line):
        lines.append(line)
        print(line, flush=True)

    shape = make_workload(args.workload).shape
    weights = rp.weights_for_engine(make_weights(shape, seed=0, device="cuda:0"))
    sets = SETS if args.sets is None else tuple(tuple(map(int, s.split(":"))) for s in args.sets.split(","))
    put(f"# The engine with its KV cache in bf16 and in 4 bits ({shape.layers} layers of {shape.n_q}/{shape.n_kv} heads of {shape.head_dim}, random weights)")
    put("")
    put("`python3 -u paper_2509_21009_amd/cache_compare.py`. Attention and append: µs in one layer of a decode step (attention with the "
        "merge of split rows; in bf16 the append is part of it).")
    put("")
    put("| rows, contexts | cache | decode step | attention | append | prefill | its attention | KV pool |")
    put("|---|---|---|---|---|---|---|---|")
    for n, lo, hi in sets:
        plens, offs, toks = _tokens(n, lo, hi, shape.vocab)
        for kv4 in (False, True):
            eng = _engine(rp, shape, weights, plens, args.new, kv4)
            step, pre, us = times(rp, eng, plens, toks, offs, args.new)
            eng.close()
            att = us[("decode", "attn")] + us.get(("decode", "attn_merge"), 0.0)
            put(" | ".join([f"| {n}, {lo:,}–{hi:,}", "4 bits" if kv4 else "bf16", f"{step:.2f} ms", f"{att:.1f} µs",
                            f"{us[('decode', 'rope_append')]:.1f} µs" if kv4 else "—", f"{pre:.0f} ms",
                            f"{us[('prefill', 'attn')]:.0f} µs", f"{rp.rp_workspace_size(eng.cfg, eng.limits)[0] / 1e9:.2f} GB |"]))
            del eng
            torch.cuda.empty_cache()
    del weights
    put("")
    put("16 prompts of 300 to 1,500 tokens, 4 given tokens each, 4,096 of the vocabulary: the largest difference of a position's logits over its "
        "largest logit, on average; the mean difference of the given token's log-probability; positions whose best token agrees.")
    put("")
    put("| first layers | logits apart | log-probability apart | same best token |")
    put("|---|---|---|---|")
    for layers in map(int, args.layers.split(",")):
        few = truncated(shape, layers, 4096)
        weights = rp.weights_for_engine(make_weights(few, seed=0, device="cuda:0"))
        plens, offs, toks = _tokens(16, 300, 1500, few.vocab)
        forced = np.random.default_rng(3).integers(0, few.vocab, (16, 4)).astype(np.int32)
        seen = []
        for kv4 in (False, True):
            eng = _engine(rp, few, weights, plens, 8, kv4)
            seen.append(logits(torch, eng, plens, toks, offs, forced))
            eng.close()
        a, b = seen
        pick = torch.from_numpy(np.roll(forced, -1, 1).T.astype(np.int64))[..., None]
        apart = (torch.log_softmax(a, -1).gather(-1, pick) - torch.log_softmax(b, -1).gather(-1, pick)).abs().mean()
        put(f"| {layers} | {((a - b).abs().amax(-1) / a.abs().amax(-1)).mean():.1%} | {apart:.4f} | {(a.argmax(-1) == b.argmax(-1)).float().mean():.0%} |")
    if args.out:
        with open(args.out, "w") as f:
            f.write("\n".join(lines) + "\n")


if __name__ == "__main__":
    main()
