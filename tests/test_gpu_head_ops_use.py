"""The operators around the head as they are used: workspaces of exactly the size asked for, streams, threads, CUDA graphs, vectors at any element, in a row
with the head and the operators on its logits."""
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_2511_12500_b200 as iris
import head_ref as ref
from test_gpu_head_ops import BF16, FP16, FP32, GUARD, KIND, check_verify, drafted, gen, near, randn, rows

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Embed:
    """Lookup and gradient; sizes that take each of the gradient's ways (few tokens, one block's sort, a cluster's)."""

    def __init__(self, n, vocab, dim, seed, dtype=BF16):
        self.n, self.vocab, self.dim, self.dtype = n, vocab, dim, dtype
        self.table = randn(vocab, dim, seed=seed).to(dtype)
        self.tokens = (torch.rand(n, device="cuda", generator=gen(seed + 1)) ** 4 * vocab).long()
        self.dy = randn(n, dim, seed=seed + 2).to(dtype)
        self.out, self.grad = torch.empty(n, dim, dtype=dtype, device="cuda"), torch.empty(vocab, dim, device="cuda")
        self.work = torch.empty(iris.iris_embed_workspace_bytes(n, vocab, dim), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        iris.iris_embed_tokens(list(self.table.chunk(2)), self.vocab, self.dim, KIND[self.dtype], self.tokens, self.n, self.out, scale=2.0, stream=stream)
        iris.iris_embed_tokens_backward(self.dy, self.n, self.dim, KIND[self.dtype], self.tokens, list(self.grad.chunk(2)), self.vocab, iris.IRIS_F32, self.work,
                                        scale=2.0, stream=stream)

    def change(self, other):
        for name in ("table", "tokens", "dy"):
            getattr(self, name).copy_(getattr(other, name))

    def outputs(self):
        return [self.out, self.grad]


class Norm:
    def __init__(self, n, dim, seed, dtype=BF16):
        self.n, self.dim, self.dtype = n, dim, dtype
        self.x, self.dy = randn(n, dim, seed=seed).to(dtype), randn(n, dim, seed=seed + 1).to(dtype)
        self.weight, self.bias = randn(dim, seed=seed + 2), randn(dim, seed=seed + 3)
        self.y, self.dx = torch.empty_like(self.x), torch.empty_like(self.x)
        self.stats, self.dw, self.db = torch.empty(n, 2, device="cuda"), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        self.work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        iris.iris_layer_norm(self.x, self.n, self.dim, KIND[self.dtype], self.y, weight=self.weight, bias=self.bias, stats=self.stats, stream=stream)
        iris.iris_layer_norm_backward(self.x, self.n, self.dim, KIND[self.dtype], self.dy, self.stats, self.work, weight=self.weight, dx=self.dx, dweight=self.dw,
                                      dbias=self.db, stream=stream)

    def change(self, other):
        for name in ("x", "dy", "weight", "bias"):
            getattr(self, name).copy_(getattr(other, name))

    def outputs(self):
        return [self.y, self.stats, self.dx, self.dw, self.db]


class Verify:
    def __init__(self, b, n, vocab, seed, dtype=BF16):
        self.b, self.n, self.vocab, self.dtype = b, n, vocab, dtype
        self.z, self.ids, self.u, self.e, self.q = drafted(b, n, vocab, dtype, seed)
        self.tokens, self.accepted = torch.empty(b, n + 1, dtype=torch.int64, device="cuda"), torch.empty(b, dtype=torch.int64, device="cuda")
        self.logprob = torch.empty(b, n + 1, device="cuda")
        self.work = torch.empty(iris.iris_verify_workspace_bytes(b, n), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        iris.iris_verify_drafts(self.z, self.b, self.n, self.vocab, KIND[self.dtype], self.ids, self.u, self.e, self.tokens, self.accepted, self.work,
                                draft_logits=self.q, logprob=self.logprob, row_stride=self.z.stride(0), draft_stride=self.q.stride(0), stream=stream)

    def change(self, other):
        for name in ("z", "ids", "u", "e", "q"):
            getattr(self, name).copy_(getattr(other, name))

    def outputs(self):
        return [self.tokens, self.accepted, self.logprob]


MAKE = {
    "embed few": lambda seed: Embed(40, 64, 100, seed), "embed": lambda seed: Embed(3000, 500, 328, seed), "embed cluster": lambda seed: Embed(12000, 2000, 64, seed, FP16),
    "norm": lambda seed: Norm(700, 1024, seed), "norm odd": lambda seed: Norm(300, 2563, seed, FP16), "norm wide": lambda seed: Norm(20, 20000, seed),
    "norm few": lambda seed: Norm(2, 5000, seed, FP32), "verify": lambda seed: Verify(6, 3, 9001, seed), "verify one": lambda seed: Verify(1, 4, 70000, seed, FP16),
}


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("what", sorted(MAKE))
def test_workspaces_are_large_enough_and_need_no_care(what):
    """Nothing behind the bytes asked for is written, and what they hold before does not matter."""
    job = MAKE[what](1)
    job.run()
    want = [t.clone() for t in job.outputs()]
    size = job.work.numel()
    for fill in (0, 0xFF):
        store = torch.full((size + 4096,), fill, dtype=torch.uint8, device="cuda")
        job.work = store[:size]
        job.run()
        assert same(job.outputs(), want) and bool((store[size:] == fill).all())


@pytest.mark.parametrize("what", sorted(MAKE))
def test_captured_calls_replay_on_other_inputs(what):
    job, other = MAKE[what](1), MAKE[what](50)
    job.run()   # eager work of the same tensors before and between
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        job.run()
        job.run()
    for source in (other, MAKE[what](90), other):
        job.change(source)
        for t in job.outputs():
            t.fill_(-3)
        graph.replay()
        got = [t.clone() for t in job.outputs()]
        job.run()
        source.run()
        assert same(got, job.outputs()) and same(got, source.outputs())


@pytest.mark.parametrize("what", sorted(MAKE))
def test_calls_on_two_streams_at_once(what):
    """Each with its own workspace; the inputs of a stream are made on it right before."""
    jobs, sources = [MAKE[what](s) for s in (1, 2)], [MAKE[what](s) for s in (30, 60)]
    for s in sources:
        s.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        for job, source, stream in zip(jobs, sources, streams):
            with torch.cuda.stream(stream):
                job.change(source)
                job.run()                       # on the current stream
                job.run(stream=stream)          # and on one that is named
    torch.cuda.synchronize()
    assert all(same(job.outputs(), source.outputs()) for job, source in zip(jobs, sources))


def test_calls_from_several_threads():
    jobs = [MAKE[what](7) for what in sorted(MAKE)]
    for job in jobs:
        job.run()
    want = [[t.clone() for t in job.outputs()] for job in jobs]
    torch.cuda.synchronize()
    errors = []

    def work(job):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    job.run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and all(same(job.outputs(), w) for job, w in zip(jobs, want))


@pytest.mark.parametrize("dim", [2563, 4096])
def test_norm_as_a_program_s_first_call(dim):
    """Shared memory beyond the usual limit is asked for by each kernel for itself: no call relies on another's having done so."""
    code = ("import torch, paper_2511_12500_b200 as iris\n"
            f"x = torch.randn(600, {dim}, device='cuda').half(); s = torch.ones(600, 2, device='cuda'); d = torch.empty_like(x); w = torch.empty({dim}, device='cuda')\n"
            f"k = torch.empty(iris.iris_layer_norm_workspace_bytes(600, {dim}), dtype=torch.uint8, device='cuda')\n"
            f"iris.iris_layer_norm_backward(x, 600, {dim}, iris.IRIS_F16, x, s, k, dx=d, dweight=w, dbias=w.clone())\n"
            "torch.cuda.synchronize(); print('done')\n")
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "done" in out.stdout, out.stderr[-2000:]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("ptype", ["rows", "fp32"])
def test_norm_with_vectors_at_any_element(dtype, ptype):
    n, dim = 9, 1003
    p = dtype if ptype == "rows" else FP32
    x, dy = randn(n, dim, seed=1).to(dtype), randn(n, dim, seed=2).to(dtype)
    for at in (1, 3):
        w, b, dw, db = (randn(dim + 8, seed=3 + i).to(p)[at:at + dim] for i in range(4))
        y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(n, 2, device="cuda")
        work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")
        iris.iris_layer_norm(x, n, dim, KIND[dtype], y, weight=w, bias=b, param_dtype=KIND[p], stats=stats)
        iris.iris_layer_norm_backward(x, n, dim, KIND[dtype], dy, stats, work, weight=w, param_dtype=KIND[p], dx=dx, dweight=dw, dbias=db)
        want, want_stats, off, off_stats = ref.norm(x, w, b, 1e-5)
        near(y, want, off, dtype)
        near(stats, want_stats, off_stats, FP32)
        want_x, want_w, want_b, off_x, off_w, off_b = ref.norm_grad(x, dy, w, stats)
        near(dx, want_x, off_x, dtype)
        near(dw, want_w, off_w, p)
        near(db, want_b, off_b, p)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_norm_of_a_column_range_next_to_another(dtype):
    """Two halves of one matrix: each call leaves the other half as it is, whatever lies there."""
    n, a, b = 40, 333, 1003
    # Rows that lie otherwise in memory are summed in another order: each way is as near the definition as its roundings allow, not the same bits.
    both = randn(n, a + b, seed=1).to(dtype)
    both[:, a:] = math.nan
    y = torch.full((n, a + b), GUARD, dtype=dtype, device="cuda")
    iris.iris_layer_norm(both[:, :a], n, a, KIND[dtype], y, row_stride=a + b, out_stride=a + b)
    want, _, off, _ = ref.norm(both[:, :a].contiguous(), None, None, 1e-5)
    near(y[:, :a], want, off, dtype)
    assert bool((y[:, a:] == GUARD).all())
    both = torch.full((n, a + b), math.inf, dtype=dtype, device="cuda")
    both[:, a:] = randn(n, b, seed=2).to(dtype)
    y = torch.full((n, a + b), GUARD, dtype=dtype, device="cuda")
    iris.iris_layer_norm(both[:, a:], n, b, KIND[dtype], y[:, a:], row_stride=a + b, out_stride=a + b)
    want, _, off, _ = ref.norm(both[:, a:].contiguous(), None, None, 1e-5)
    near(y[:, a:], want, off, dtype)
    assert bool((y[:, :a] == GUARD).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,dim,stride,shift", [(300, 1, 1, 0), (300, 1, 1, 3), (40, 3, 4, 1), (40, 5, 7, 2), (40, 7, 7, 1), (40, 8, 9, 5)])
def test_norm_of_rows_shorter_than_16_bytes(dtype, n, dim, stride, shift):
    """Several rows in the same 16 bytes; around the matrix nothing counts, whatever lies there."""
    def matrix(seed):
        store = torch.full((n * stride + 64,), math.nan, dtype=dtype, device="cuda")
        view = store[shift:].as_strided((n, dim), (stride, 1), shift)
        view.copy_(randn(n, dim, seed=seed))
        return view

    x, dy, w = matrix(1), matrix(2), randn(dim, seed=3)
    y, dx, stats, dw = matrix(4), matrix(5), torch.empty(n, 2, device="cuda"), torch.empty(dim, device="cuda")
    work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")
    iris.iris_layer_norm(x, n, dim, KIND[dtype], y, weight=w, stats=stats, eps=0.5, row_stride=stride, out_stride=stride)
    iris.iris_layer_norm_backward(x, n, dim, KIND[dtype], dy, stats, work, weight=w, dx=dx, dweight=dw, row_stride=stride, dy_stride=stride, dx_stride=stride)
    want, _, off, _ = ref.norm(x, w, None, 0.5)
    near(y, want, off, dtype)
    want_x, want_w, _, off_x, off_w, _ = ref.norm_grad(x, dy, w, stats)
    near(dx, want_x, off_x, dtype)
    near(dw, want_w, off_w, FP32)


def test_verify_drafts_end_at_the_first_that_is_absent():
    b, n, vocab = 8, 4, 500
    z, t, u, e, q = drafted(b, n, vocab, BF16, 11, agree=0.1)
    u.zero_()                     # everything that can be is accepted
    t[0, 1] = -1
    t[1, 0] = vocab
    t[2, 3] = 1 << 40
    t[3] = -5
    tokens, accepted = torch.empty(b, n + 1, dtype=torch.int64, device="cuda"), torch.empty(b, dtype=torch.int64, device="cuda")
    work = torch.empty(iris.iris_verify_workspace_bytes(b, n), dtype=torch.uint8, device="cuda")
    iris.iris_verify_drafts(z, b, n, vocab, iris.IRIS_BF16, t, u, e, tokens, accepted, work, draft_logits=q)
    assert accepted.tolist() == [1, 0, 3, 0, 4, 4, 4, 4]
    for i in range(b):
        a = int(accepted[i])
        assert tokens[i, :a].tolist() == t[i, :a].tolist() and 0 <= int(tokens[i, a]) < vocab and bool((tokens[i, a + 1:] == -1).all())
    check_verify(z, n, t, u, e, q)


def test_the_greedy_way_without_random_numbers():
    z = randn(12, 3000, seed=1)
    best = z.view(4, 3, 3000).argmax(2)
    ids = best[:, :2].clone()
    ids[2, 1] += 1
    tokens, accepted = torch.empty(4, 3, dtype=torch.int64, device="cuda"), torch.empty(4, dtype=torch.int64, device="cuda")
    work = torch.empty(iris.iris_verify_workspace_bytes(4, 2), dtype=torch.uint8, device="cuda")
    iris.iris_verify_drafts(z, 4, 2, 3000, iris.IRIS_F32, ids, None, None, tokens, accepted, work, scale=math.inf)
    assert accepted.tolist() == [2, 2, 1, 2]
    assert tokens[2].tolist() == [int(best[2, 0]), int(best[2, 1]), -1] and torch.equal(tokens[[0, 1, 3]], best[[0, 1, 3]])


class Model:
    """Tied embeddings in `world` shards on the heap, a norm, the head."""

    def __init__(self, world, vocab, dim, tokens, seed, soft=4.0):
        self.world, self.vocab, self.dim, self.tokens = world, vocab, dim, tokens
        self.heap = iris.iris_heap_create(world, iris.iris_gemm_heap_bytes(tokens, vocab, world))
        self.table = (randn(vocab, dim, seed=seed) * (soft / dim ** 0.5)).bfloat16()
        self.shards = list(self.table.chunk(world))
        self.weight, self.bias = 1 + 0.1 * randn(dim, seed=seed + 1), 0.1 * randn(dim, seed=seed + 2)
        self.e, self.h = (torch.empty(tokens, dim, dtype=BF16, device="cuda") for _ in range(2))
        self.stats = torch.empty(tokens, 2, device="cuda")

    def forward(self, ids):
        n = ids.numel()
        iris.iris_embed_tokens(self.shards, self.vocab, self.dim, iris.IRIS_BF16, ids, n, self.e, scale=self.dim ** 0.5)
        iris.iris_layer_norm(self.e, n, self.dim, iris.IRIS_BF16, self.h, weight=self.weight, bias=self.bias, stats=self.stats)
        iris.gemm_all_scatter(self.h, self.shards, self.heap, self.tokens, self.vocab, self.dim, self.world, iris.IRIS_MODE_FUSED_SEQUENTIAL)
        return iris.iris_heap_base(self.heap, self.world - 1)

    def logits(self):
        z = torch.empty(self.tokens, self.vocab, dtype=BF16, device="cuda")
        iris.iris_load_tile(self.heap, iris.iris_heap_base(self.heap, self.world - 1), z, self.tokens, self.vocab * 2, self.vocab * 2, self.vocab * 2,
                            self.world - 1, self.world - 1)
        return z

    def close(self):
        iris.iris_heap_destroy(self.heap)


def test_a_serving_step():
    """ids -> lookup -> norm -> head -> verification of drafts on the logits in a slot -> ids -> lookup."""
    b, n, vocab, dim = 16, 3, 2048, 256
    model = Model(2, vocab, dim, b * (n + 1), 3)
    try:
        ids = torch.randint(0, vocab, (b * (n + 1),), device="cuda", generator=gen(8))
        at = model.forward(ids)
        z = model.logits()
        e = (model.table[ids].float() * float(torch.tensor(dim ** 0.5))).bfloat16()
        assert torch.equal(model.e, e)
        want, _, off, _ = ref.norm(model.e, model.weight, model.bias, 1e-5)
        near(model.h, want, off, BF16)
        want = model.h.double() @ model.table.double().t()
        assert bool(((z.double() - want).abs() <= 2.0 ** -8 * want.abs() + dim * ref.F32 * (model.h.double().abs() @ model.table.double().abs().t())).all())
        q = (z.view(b, n + 1, vocab)[:, :n].reshape(b * n, vocab).float() + randn(b * n, vocab, seed=4)).bfloat16()
        race = torch.empty(b * n, vocab, device="cuda").exponential_(generator=gen(5))
        drafts = (q.float() - race.log()).argmax(1).view(b, n)
        u, noise = torch.rand(b, n, device="cuda", generator=gen(6)), torch.empty(b, vocab, device="cuda").exponential_(generator=gen(7))
        tokens, accepted = torch.empty(b, n + 1, dtype=torch.int64, device="cuda"), torch.empty(b, dtype=torch.int64, device="cuda")
        work = torch.empty(iris.iris_verify_workspace_bytes(b, n), dtype=torch.uint8, device="cuda")
        iris.iris_verify_drafts(at, b, n, vocab, iris.IRIS_BF16, drafts, u, noise, tokens, accepted, work, draft_logits=q)
        check_verify(z, n, drafts, u, noise, q)
        again = torch.empty_like(tokens)
        iris.iris_verify_drafts(z, b, n, vocab, iris.IRIS_BF16, drafts, u, noise, again, accepted, work, draft_logits=q)
        assert torch.equal(tokens, again)
        nxt = torch.empty(b * (n + 1), dim, dtype=BF16, device="cuda")   # places behind the next token have rows of 0
        iris.iris_embed_tokens(model.shards, vocab, dim, iris.IRIS_BF16, tokens, b * (n + 1), nxt)
        flat = tokens.flatten()
        assert torch.equal(nxt, model.table[flat.clamp(min=0)] * (flat >= 0)[:, None])
    finally:
        model.close()


def test_the_gradients_of_a_training_step():
    """-sum of the next tokens' log probabilities, its gradient for the tied table and the norm's vectors against 64-bit autograd on the same values.  Six roundings
    to bf16 on the way (lookup, norm, logits, their gradient, its product, the norm's gradient) are off by at most 2^-8 each and mostly by a third of that,
    logits of up to about 8 by 2^-5: 3 % of the gradients' norms."""
    n, vocab, dim = 512, 1024, 192
    model = Model(2, vocab, dim, n, 5, soft=1.0)
    try:
        ids = (torch.rand(n, device="cuda", generator=gen(1)) ** 3 * vocab).long()
        nxt = torch.randint(0, vocab, (n, 1), device="cuda", generator=gen(2))
        at = model.forward(ids)
        f32 = dict(device="cuda")
        lp, stats, dz = torch.empty(n, 1, **f32), torch.empty(n, 2, **f32), torch.empty(n, vocab, dtype=BF16, device="cuda")
        iris.iris_token_logprobs(at, n, vocab, iris.IRIS_BF16, targets=nxt, n_targets=1, logprob=lp, stats=stats)
        iris.iris_token_logprobs_backward(at, n, vocab, iris.IRIS_BF16, nxt, 1, stats, -torch.ones(n, 1, **f32), dz)
        dh = (dz @ model.table).contiguous()
        dtable = torch.empty(vocab, dim, **f32)
        dx, dw, db = torch.empty_like(dh), torch.empty(dim, **f32), torch.empty(dim, **f32)
        work = torch.empty(max(iris.iris_layer_norm_workspace_bytes(n, dim), iris.iris_embed_workspace_bytes(n, vocab, dim)), dtype=torch.uint8, device="cuda")
        iris.iris_layer_norm_backward(model.e, n, dim, iris.IRIS_BF16, dh, model.stats, work, weight=model.weight, dx=dx, dweight=dw, dbias=db)
        dtable.copy_((dz.t() @ model.h).float())   # the head's share; the lookup's is added
        iris.iris_embed_tokens_backward(dx, n, dim, iris.IRIS_BF16, ids, list(dtable.chunk(2)), vocab, iris.IRIS_F32, work, scale=dim ** 0.5, accumulate=True)

        t, w, c = (v.double().requires_grad_() for v in (model.table, model.weight, model.bias))
        e = t[ids] * float(torch.tensor(dim ** 0.5))
        h = torch.nn.functional.layer_norm(e, (dim,), w, c, 1e-5)
        loss = -torch.log_softmax(h @ t.t(), 1).gather(1, nxt).sum()
        loss.backward()
        assert abs(float(-lp.double().sum() - loss.detach())) < 0.01 * float(loss.detach())
        for got, want in ((dtable, t.grad), (dw, w.grad), (db, c.grad)):
            assert float((got.double() - want).norm()) < 0.03 * float(want.norm())
    finally:
        model.close()
