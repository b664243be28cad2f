"""The local step's operators where something is shared: one row by most tokens, one workspace by calls without a wait between
them, one handle by threads and streams; and that nothing is left over or allocated by a call."""

import math
import threading

import pytest
import torch

import test_gpu_lm_ops as base
from test_gpu_lm_ops import BF16, E24, F16, F32, embed_grad_ref, gen, randn, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ops(B):
    o = B.LmOps(0)
    yield o
    assert o.cocodc_lm_poll_status() == B.OK
    o.close()


# ------------------------------------------------------------------------------------------- one row by most tokens

def ids_of(kind, T, V, g):
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind == "padding at the end":                          # a third of the places hold id 0
        ids[2 * T // 3:] = 0
    elif kind == "padding here and there":
        ids[torch.rand(T, generator=g, device="cuda") < 0.35] = 0
    elif kind == "one id":
        ids.fill_(V - 1)
    elif kind == "two ids, turn about":
        ids[0::2], ids[1::2] = 3, 3 + 128                     # both in one bin where there are 128 bins
    elif kind == "one bin":                                   # every 128th row
        ids = ids // 128 * 128
    elif kind == "just below a full list":                    # 384 hits in 2048 ids, and one more in the next 2048
        ids = torch.where(ids == 5, ids + 1, ids)
        ids.view(-1)[:384] = 5
        ids.view(-1)[T // 32:T // 32 + 385] = 5
    return ids


@pytest.mark.parametrize("kind", ["padding at the end", "padding here and there", "one id", "two ids, turn about", "one bin", "just below a full list"])
@pytest.mark.parametrize("T,V,D", [(65536, 32000, 24), (65536, 300, 16), (16411, 50257, 33)])
def test_embed_grad_of_frequent_tokens(ops, kind, T, V, D):
    """More tokens of one bin than a warp's list holds: the ids are walked a second time."""
    g = gen(T + V)
    ids = ids_of(kind, T, V, g).clamp_(max=V - 1)
    dy = randn(g, T, D, dtype=BF16)
    ref, bound = embed_grad_ref(dy, ids, V, 0.5)
    for index in (torch.int32, torch.int64):
        got = torch.full((V, D), math.nan, device="cuda")
        ops.cocodc_lm_embed_grad(dy, ids.to(index), got, scale=0.5)
        within(got, ref, bound, kind)
        again = torch.empty_like(got)
        ops.cocodc_lm_embed_grad(dy, ids.to(index), again, scale=0.5)
        assert torch.equal(again, got)
    start = randn(g, V, D)
    acc = start.clone()
    ops.cocodc_lm_embed_grad(dy, ids, acc, scale=0.5, accumulate=True)
    within(acc, ref + start.double(), bound + E24 * start.abs().double(), "accumulated")


@pytest.mark.parametrize("T,V,D", [(1, 4000, 64), (500, 300, 768), (257, 129, 77), (4099, 1000, 136)])
@pytest.mark.parametrize("table", [BF16, F16, F32])
@pytest.mark.parametrize("grad", [BF16, F32])
def test_accumulate_into_a_table_of_any_type(ops, T, V, D, table, grad):
    """Added in fp32 to what the table holds, rounded once; rows of tokens that do not occur keep their bits."""
    g = gen(T + D)
    dy = randn(g, T, D, dtype=grad)
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda")
    ref, bound = embed_grad_ref(dy, ids, V, 1.5)
    start = randn(g, V, D, dtype=table)
    got = start.clone()
    ops.cocodc_lm_embed_grad(dy, ids, got, scale=1.5, accumulate=True)
    within(got, ref + start.double(), bound + E24 * start.double().abs(), "accumulated")
    named = torch.bincount(ids[ids >= 0], minlength=V) > 0
    assert torch.equal(got[~named], start[~named])


@pytest.mark.parametrize("T,D,F", [(1, 1, 1), (7, 1000, 264), (33, 320, 416), (129, 192, 384), (200, 33, 65), (300, 264, 520)])
def test_glu_grad_silu_in_half_precision(ops, T, D, F):
    base.test_glu_grad(ops, T, D, F, F16, "silu")


# ------------------------------------------------------------------------------------------- a step's calls, and their inputs

class Step:
    """Inputs of one call of each operator, of odd and even sizes by the seed, and a run of them with outputs of its own."""

    def __init__(self, ops, seed):
        g = gen(seed)
        self.ops = ops
        # up to three tiles of rows, whose dx goes in parts where F is long; now and then rows off 16 bytes
        T, D, F, V = 5 + 61 * (seed % 5), (64, 72, 33)[seed % 3], (2048, 520, 65)[seed % 3], (700, 33, 5003)[seed % 3]
        self.table, self.ids = randn(g, V, D), torch.randint(-1, V, (T,), generator=g, device="cuda")
        self.x, self.dh = randn(g, T, D, dtype=BF16), randn(g, T, F, dtype=BF16)
        self.wg, self.wu = (randn(g, F, D, std=D ** -0.5, dtype=BF16) for _ in range(2))
        self.logits, self.targets = randn(g, T, 4 * V, std=3.0, dtype=BF16), torch.randint(0, 4 * V, (T,), generator=g, device="cuda")
        self.one = torch.ones(T, device="cuda")
        self.sizes = (V, D, T), (T, D, F)
        self.shapes = dict(y=((T, D), BF16), h=((T, F), BF16), gate=((T, F), BF16), up=((T, F), BF16), dx=((T, D), BF16), dwg=((F, D), BF16),
                           dwu=((F, D), BF16), dtable=((V, D), F32), logp=((T,), F32), entropy=((T,), F32), lse=((T,), F32),
                           top=((T, 4), torch.int32), top_logp=((T, 4), F32), dlogits=((T, 4 * V), BF16))

    def outputs(self):
        return {n: torch.zeros(s, dtype=t, device="cuda") for n, (s, t) in self.shapes.items()}

    def workspaces(self, B):
        lib = B.library()
        return lib.cocodc_lm_embed_grad_workspace(*self.sizes[0]), lib.cocodc_lm_glu_grad_workspace(*self.sizes[1])

    def run(self, o, workspace=None):
        ops = self.ops
        ops.cocodc_lm_embed(self.table, self.ids, o["y"], scale=2.0)
        ops.cocodc_lm_glu(self.x, self.wg, self.wu, o["h"], gate=o["gate"], up=o["up"])
        ops.cocodc_lm_glu_grad(self.dh, o["gate"], o["up"], self.x, self.wg, self.wu, o["dx"], o["dwg"], o["dwu"], workspace=workspace)
        ops.cocodc_lm_embed_grad(o["dx"], self.ids, o["dtable"], scale=2.0, workspace=workspace)
        ops.cocodc_lm_logprobs(self.logits, self.targets, o["logp"], entropy=o["entropy"], lse=o["lse"], top_ids=o["top"], top_logp=o["top_logp"])
        ops.cocodc_lm_logprobs_grad(self.logits, self.targets, o["lse"], o["entropy"], self.one, self.one, o["dlogits"])
        return o


def same(a, b):
    return all(torch.equal(a[n], b[n]) for n in a)


def test_one_workspace_for_calls_without_a_wait_between_them(B, ops):
    """Alternating sizes; every kernel starts before the one ahead of it, which may still read the workspace, has ended.  The
    workspace starts full of NaN."""
    steps = [Step(ops, s) for s in range(15)]
    want = [s.run(s.outputs()) for s in steps]
    work = torch.empty(max(max(s.workspaces(B)) for s in steps), dtype=torch.uint8, device="cuda")
    for _ in range(4):
        got = [s.outputs() for s in steps]
        work.fill_(255)
        torch.cuda.synchronize()
        for s, o in zip(steps, got):
            s.run(o, work)
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(want, got))


def test_one_handle_on_two_streams_from_two_threads(B, ops):
    steps = [Step(ops, s) for s in range(24)]
    want = [s.run(s.outputs()) for s in steps]
    rounds = 6
    got = [[s.outputs() for s in steps] for _ in range(rounds)]
    work = [torch.empty(max(max(s.workspaces(B)) for s in steps), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    failed, before = [], ops.launch_count

    def worker(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for r in range(rounds):
                    for s, o in list(zip(steps, got[r]))[k::2]:
                        s.run(o, work[k])
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=worker, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(same(a, b) for r in got for a, b in zip(want, r))
    launches = ops.launch_count - before
    assert launches % rounds == 0
    at = ops.launch_count
    for s, o in zip(steps, got[0]):
        s.run(o, work[0])
    assert ops.launch_count - at == launches // rounds        # none lost by counting from two threads
    torch.cuda.synchronize()


def test_calls_with_a_workspace_allocate_nothing(B, ops):
    step = Step(ops, 4)
    o, work = step.outputs(), torch.empty(max(step.workspaces(B)), dtype=torch.uint8, device="cuda")
    step.run(o, work)
    torch.cuda.synchronize()
    count, free = torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.mem_get_info()[0]
    for _ in range(20):
        step.run(o, work)
    torch.cuda.synchronize()
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == count
    assert torch.cuda.mem_get_info()[0] >= free - (1 << 21)
