"""Run one kernel of the search on a chosen range, for timing and profiling.

  python -m paper_2607_22242_gb300.profile_case --kernel search --config 3 --count 67108864 --reps 3
  python -m paper_2607_22242_gb300.profile_case --kernel eval --config 2 --count 16777216
  python -m paper_2607_22242_gb300.profile_case --kernel batch --batch 1024
  python -m paper_2607_22242_gb300.profile_case --kernel list --config 3 --count 16777216
  python -m paper_2607_22242_gb300.profile_case --kernel whatif --config 3 --reps 20
  python -m paper_2607_22242_gb300.profile_case --kernel tree --workload wide32 --space 3
  python -m paper_2607_22242_gb300.profile_case --kernel policy --rows 1024 --vocab 131072 --dtype bfloat16
  python -m paper_2607_22242_gb300.profile_case --kernel attention --beams 64 --prefix 65536 --suffix 512

Prints one line per repetition (CUDA-event time of the call and mappings/s; for the learning calls -- policy,
preference, scores, embed_grad -- and the answering calls -- attention, beams, reorder -- GB/s of the bytes they
cannot do without).
Sized so that a profiler capture of one launch stays short.
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def learning_call(args):
    """(bytes that it cannot do without, the call) of a learning entry point on random inputs, answers of 16 tokens."""
    import torch
    from paper_2607_22242_gb300 import bf
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = getattr(torch, args.dtype)
    size = torch.empty(0, dtype=dtype).element_size()
    tokens = torch.randint(args.vocab, (args.rows,), generator=gen, device="cuda")
    if args.kernel == "embed_grad":
        grad = torch.randn(args.rows, args.width, generator=gen, device="cuda").to(dtype)
        return (args.rows + args.vocab) * args.width * size, lambda: bf.embed_grad(grad, tokens, args.vocab)
    logits = torch.randn(args.rows, args.vocab, generator=gen, device="cuda", dtype=torch.float32).mul_(2).to(dtype)
    moved = args.rows * args.vocab * size
    if args.kernel == "scores":
        return moved, lambda: bf.token_logprobs(logits, tokens, entropy=True)
    old = bf.token_logprobs(logits, tokens)
    answers = max(2, args.rows // 32 * 2)
    offsets = torch.linspace(0, args.rows, answers + 1, device="cuda").round().long()
    if args.kernel == "preference":
        return 2 * moved, lambda: bf.preference_loss(logits, tokens, offsets, old)
    advantage = torch.randn(answers, generator=gen, device="cuda")
    return 2 * moved, lambda: bf.policy_loss(logits, tokens, offsets, old, advantage, old, kl_coef=0.04)


def answering_call(args):
    """(bytes that it cannot do without, the call) of an answering entry point on random inputs."""
    import torch
    from paper_2607_22242_gb300 import bf
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = getattr(torch, args.dtype)
    size = torch.empty(0, dtype=dtype).element_size()
    randn = lambda *n: torch.randn(*n, generator=gen, device="cuda", dtype=dtype)
    rows, heads, dim = args.groups * args.beams, args.kv_heads, args.dim
    if args.kernel == "beams":
        logits, scores = randn(rows, args.vocab), torch.randn(rows, generator=gen, device="cuda")
        return rows * args.vocab * size, lambda: bf.beam_step(logits, scores, args.beams, keep=args.keep)
    if args.kernel == "reorder":  # every second row of a group is written from the one before it
        parents = torch.arange(rows, device="cuda") // 2 * 2
        states = [randn(rows, args.suffix, heads, dim) for _ in range(8)]
        moved = 8 * (rows // 2) * 2 * args.suffix * heads * dim * size
        return moved, lambda: bf.beam_reorder(states, parents, args.beams)
    q = randn(rows, heads * args.share, dim)
    prefix = [randn(args.groups, args.prefix, heads, dim) for _ in range(2)]
    suffix = [randn(rows, args.suffix, heads, dim) for _ in range(2)]
    moved = 2 * (args.groups * args.prefix + rows * args.suffix) * heads * dim * size + 2 * q.numel() * size
    return moved, lambda: bf.prefix_attention(q, *prefix, *suffix)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--kernel", choices=("search", "pruned", "eval", "batch", "list", "whatif", "tree",
                                             "policy", "preference", "scores", "embed_grad",
                                             "attention", "beams", "reorder"), default="search")
    ap.add_argument("--config", type=int, default=3)
    ap.add_argument("--workload", default=None, help="wide28 | wide32 | layered24 (instead of --config)")
    ap.add_argument("--space", type=int, default=3, help="tree search: 3 = full space, 2 = binary")
    ap.add_argument("--no-prune", action="store_true", help="tree search: simulate every mapping")
    ap.add_argument("--first", type=int, default=0)
    ap.add_argument("--count", type=int, default=1 << 26)
    ap.add_argument("--batch", type=int, default=1024, help="scenarios for --kernel batch (config 4 prefix)")
    ap.add_argument("--reps", type=int, default=3)
    ap.add_argument("--rows", type=int, default=1024, help="learning calls: tokens")
    ap.add_argument("--vocab", type=int, default=32768)
    ap.add_argument("--width", type=int, default=2048, help="embed_grad: columns of the table")
    ap.add_argument("--groups", type=int, default=1, help="answering calls: prompts")
    ap.add_argument("--beams", type=int, default=16, help="answers of a prompt")
    ap.add_argument("--keep", type=int, default=16, help="beams: continuations")
    ap.add_argument("--prefix", type=int, default=8192, help="attention: tokens of a prompt")
    ap.add_argument("--suffix", type=int, default=256, help="attention, reorder: tokens of an answer")
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--share", type=int, default=4, help="attention: query heads of a key head")
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--dtype", default="bfloat16", choices=("float32", "bfloat16", "float16"))
    args = ap.parse_args()

    import torch
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_22242_gb300 import bf
    from paper_2607_22242_gb300 import scenarios as S

    torch.cuda.set_device(0)
    stream = torch.cuda.current_stream()
    unit = "mappings/s"
    if args.kernel in ("policy", "preference", "scores", "embed_grad"):
        work, call = learning_call(args)
        unit = "B/s"
    elif args.kernel in ("attention", "beams", "reorder"):
        work, call = answering_call(args)
        unit = "B/s"
    elif args.kernel == "batch":
        batch = S.config4(args.batch)
        work = len(batch) * 3 ** 10
        packed = bf.pack_descs(batch)  # the C caller's desc array, packed once
        call = lambda: bf.search_batch(batch, stream, packed)
    else:
        scn = getattr(S, args.workload)() if args.workload else S.config(args.config)
        count = min(args.count, 3 ** scn.n - args.first)
        work = count
        h = bf.create_scenario(scn)
        if args.kernel == "tree":  # branch and bound over the chosen space (count ignored)
            work = args.space ** scn.n
            stats = {}

            def call():
                res, st = bf.search_tree(h, args.space, not args.no_prune, None, stream)
                stats.update(st)
                return res
        elif args.kernel == "search":
            call = lambda: bf.search_range(h, args.first, count, stream)
        elif args.kernel == "pruned":  # branch and bound over the whole space (count ignored)
            work = 3 ** scn.n
            call = lambda: bf.search_pruned(h, None, stream)
        elif args.kernel == "list":  # uniformly random mapping indices of the whole space
            g = torch.Generator(device="cuda").manual_seed(1)
            idx = torch.randint(0, 3 ** scn.n, (count,), device="cuda", generator=g, dtype=torch.int64)
            ms = torch.empty(count, dtype=torch.int32, device="cuda")
            fe = torch.empty(count, dtype=torch.uint8, device="cuda")
            call = lambda: bf.eval_indices(h, idx, ms, fe, stream)
        elif args.kernel == "whatif":  # around the optimum of the scenario
            base = bf.search_best(h, stream).index
            work = len(bf.whatif(h, base, stream))
            call = lambda: bf.whatif(h, base, stream)
        else:
            ms = torch.empty(count, dtype=torch.int32, device="cuda")
            fe = torch.empty(count, dtype=torch.uint8, device="cuda")
            call = lambda: bf.eval_mappings(h, args.first, count, ms, fe, stream)
    for rep in range(args.reps):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record(stream)
        out = call()
        b.record(stream)
        b.synchronize()
        t = a.elapsed_time(b)
        print(f"{args.kernel} rep {rep}: {t:.3f} ms, {work / (t / 1e3):.4g} {unit}"
              + (f", best {out.index}/{out.makespan_us}" if args.kernel in ("search", "pruned", "tree") else "")
              + (f", {stats}" if args.kernel == "tree" else ""), flush=True)


if __name__ == "__main__":
    main()
