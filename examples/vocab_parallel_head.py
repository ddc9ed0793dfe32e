"""A vocabulary-parallel LM head on the symmetric heap, and what follows it: scores of the next tokens and one distillation step.

Every rank holds a column shard of the output embedding.  gemm_all_scatter leaves all logits in every rank's slot; the rows are then shared out,
and each rank scores and distils its own rows from its own slot:

    teacher's logits --> the 64 largest of each row with their log probabilities          iris_token_logprobs
    student's logits --> log probability of the next token, entropy                       iris_token_logprobs
                     --> loss against the teacher's list and, in place, its gradient      iris_distill_topk
                     --> gradient of the summed log probabilities (policy gradient)       iris_token_logprobs_backward

    python examples/vocab_parallel_head.py [--world 8] [--tokens 2048] [--vocab 32768] [--hidden 2048] [--list 64]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_12500_b200 as iris  # noqa: E402


class Head:
    """A head's heap: W emulated ranks, each with a copy of the logits [tokens, vocab] at offset 0 of its slot."""

    def __init__(self, world: int, tokens: int, vocab: int):
        self.world, self.tokens, self.vocab = world, tokens, vocab
        self.handle = iris.iris_heap_create(world, iris.iris_gemm_heap_bytes(tokens, vocab, world))

    def logits(self, hidden: torch.Tensor, shards: list[torch.Tensor]):
        """hidden [tokens, d] bf16, shards [vocab / world, d] bf16."""
        iris.gemm_all_scatter(hidden, shards, self.handle, self.tokens, self.vocab, hidden.shape[1], self.world, iris.IRIS_MODE_FUSED_SEQUENTIAL)

    def rows_of(self, rank: int) -> tuple[int, int, int]:
        """(device address, first row, number of rows) of rank's share in rank's own slot."""
        a, b = self.tokens * rank // self.world, self.tokens * (rank + 1) // self.world
        return iris.iris_heap_base(self.handle, rank) + a * self.vocab * 2, a, b - a

    def close(self):
        iris.iris_heap_destroy(self.handle)


def step(teacher: Head, student: Head, next_token: torch.Tensor, weight: torch.Tensor, k: int) -> dict[str, torch.Tensor]:
    """What a training step needs of the two heads' logits, rank by rank.  The student's own rows become d loss / d logits in their slots."""
    n, f32 = student.tokens, dict(dtype=torch.float32, device="cuda")
    out = dict(ids=torch.empty(n, k, dtype=torch.int64, device="cuda"), teacher=torch.empty(n, k, **f32), logprob=torch.empty(n, 1, **f32),
               entropy=torch.empty(n, **f32), stats=torch.empty(n, 2, **f32), loss=torch.empty(n, **f32),
               policy=torch.empty(n, student.vocab, dtype=torch.bfloat16, device="cuda"))
    ones = torch.ones(n, 1, **f32)
    for rank in range(student.world):
        at, r, rows = teacher.rows_of(rank)
        iris.iris_token_logprobs(at, rows, teacher.vocab, iris.IRIS_BF16, top_k=k, top_ids=out["ids"][r:], top_logprob=out["teacher"][r:])
        at, r, rows = student.rows_of(rank)
        iris.iris_token_logprobs(at, rows, student.vocab, iris.IRIS_BF16, targets=next_token[r:], n_targets=1, logprob=out["logprob"][r:],
                                 entropy=out["entropy"][r:], stats=out["stats"][r:])
        iris.iris_token_logprobs_backward(at, rows, student.vocab, iris.IRIS_BF16, next_token[r:], 1, out["stats"][r:], ones[r:], out["policy"][r:])
        iris.iris_distill_topk(at, rows, student.vocab, iris.IRIS_BF16, out["teacher"][r:], out["ids"][r:], k, out["loss"][r:],
                               mode=iris.IRIS_DISTILL_TAIL, weight=weight[r:], dlogits=at)
    return out


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--world", type=int, default=8)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--vocab", type=int, default=32768)
    p.add_argument("--hidden", type=int, default=2048)
    p.add_argument("--list", type=int, default=64)
    a = p.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(0)
    hidden = torch.randn(a.tokens, a.hidden, device="cuda", generator=gen).bfloat16()
    embed = [torch.randn(a.vocab // a.world, a.hidden, device="cuda", generator=gen).mul_(2 / a.hidden ** 0.5).bfloat16() for _ in range(a.world)]
    better = [(e + 0.2 * torch.randn(e.shape, device="cuda", generator=gen) / a.hidden ** 0.5).bfloat16() for e in embed]
    next_token = torch.randint(0, a.vocab, (a.tokens, 1), device="cuda", generator=gen)
    weight = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")
    teacher, student = Head(a.world, a.tokens, a.vocab), Head(a.world, a.tokens, a.vocab)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    try:
        for _ in range(3):
            teacher.logits(hidden, better)
            student.logits(hidden, embed)
            begin.record()
            out = step(teacher, student, next_token, weight, a.list)
            end.record()
            torch.cuda.synchronize()
        print(f"loss {out['loss'].mean().item():.5f}  entropy {out['entropy'].mean().item():.4f}  log probability {out['logprob'].mean().item():.4f}  "
              f"{begin.elapsed_time(end) * 1e3:.0f} us for {a.world} ranks' rows")
    finally:
        teacher.close()
        student.close()


if __name__ == "__main__":
    main()
