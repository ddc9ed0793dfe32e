"""The head example: logits from gemm_all_scatter in every slot, then scores, the teacher's list, loss and gradient of each rank's own rows."""
import os
import sys

import numpy as np
import pytest
import torch

import logit_ref as ref
import paper_2511_12500_b200 as iris

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import vocab_parallel_head as head  # noqa: E402

pytestmark = pytest.mark.gpu


def slot(h, rank):
    """Rank's copy of the logits as a tensor of this process."""
    out = torch.empty(h.tokens, h.vocab, dtype=torch.bfloat16, device="cuda")
    iris.iris_load_tile(h.handle, iris.iris_heap_base(h.handle, rank), out, h.tokens, h.vocab * 2, h.vocab * 2, h.vocab * 2, rank, rank)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("world,tokens,vocab,d,k", [(2, 24, 512, 64, 8), (4, 50, 4096, 128, 64)])
def test_head_step(world, tokens, vocab, d, k):
    gen = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn(tokens, d, device="cuda", generator=gen).bfloat16()
    shards = [[(2 * torch.randn(vocab // world, d, device="cuda", generator=gen) / d ** 0.5).bfloat16() for _ in range(world)] for _ in range(2)]
    nxt = torch.randint(0, vocab, (tokens, 1), device="cuda", generator=gen)
    weight = torch.rand(tokens, device="cuda", generator=gen)
    teacher, student = head.Head(world, tokens, vocab), head.Head(world, tokens, vocab)
    try:
        teacher.logits(hidden, shards[0])
        student.logits(hidden, shards[1])
        zt, zs = slot(teacher, world - 1), slot(student, world - 1)
        want = hidden.double() @ torch.cat(shards[1]).double().T
        assert float((zs.double() - want).abs().max()) <= 1e-2 * (float(want.abs().max()) + 1)
        out = head.step(teacher, student, nxt, weight, k)
        torch.cuda.synchronize()
        for rank in range(world):
            a, b = tokens * rank // world, tokens * (rank + 1) // world
            mine = slot(student, rank)
            assert torch.equal(mine[:a], zs[:a]) and torch.equal(mine[b:], zs[b:])          # other ranks' rows stay logits
            for r in range(a, b):
                t, s = zt[r].double().cpu().numpy(), zs[r].double().cpu().numpy()
                lt, ls = ref.log_softmax(t, 1.0)[2], ref.log_softmax(s, 1.0)[2]
                ids = ref.top(t, k)
                assert np.array_equal(out["ids"][r].cpu().numpy(), ids)
                assert np.allclose(out["teacher"][r].cpu().numpy(), lt[ids], atol=2e-5)
                j = int(nxt[r, 0])
                assert abs(out["logprob"][r, 0].item() - ls[j]) < 2e-5 and abs(out["entropy"][r].item() - ref.entropy(ls)) < 5e-5
                policy = -np.exp(ls)
                policy[j] += 1
                assert np.all(np.abs(out["policy"][r].double().cpu().numpy() - policy) <= 2.0 ** -8 * np.abs(policy) + 1e-5)
                loss, dz, size, dsize, _ = ref.distill(s, 1.0, ids, out["teacher"][r].cpu().numpy(), 1.0, True)
                assert abs(out["loss"][r].item() - loss) < 1e-5 + 1e-5 * size
                w = float(weight[r])
                assert np.all(np.abs(mine[r].double().cpu().numpy() - w * dz) <= 2.0 ** -8 * np.abs(w * dz) + 3e-5 * w * dsize + 1e-37)
    finally:
        teacher.close()
        student.close()


def test_the_command_runs(capsys):
    head.main(["--world", "2", "--tokens", "64", "--vocab", "1024", "--hidden", "64", "--list", "16"])
    assert "loss" in capsys.readouterr().out
