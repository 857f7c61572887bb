"""Clipping of gradients that two gloo ranks hold in part: the host side of sharded.clip_over_ranks (one all-reduce of the
sums of squares), with the library's two calls replaced by their definitions in torch."""
import math
import os

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp


class PlainKernels:
    """Stand-in for gc_grad_norm and gc_grad_scale, written from their documented contract."""

    def grad_sq_sum(self, grads, sq_sum, ws, dev_status):
        sq_sum[0] = sum(float((g.double() ** 2).sum()) for g in grads)
        self._flag(sq_sum, dev_status)

    def grad_scale(self, grads, sq_sum, max_norm, dev_status):
        self._flag(sq_sum, dev_status)
        if math.isfinite(sq_sum.item()):
            for g in grads:
                g.mul_(min(1.0, max_norm / (math.sqrt(sq_sum.item()) + 1e-6)))

    def _flag(self, sq_sum, dev_status):
        if not math.isfinite(sq_sum.item()):
            dev_status |= 8


def _parts(rank):
    gen = torch.Generator().manual_seed(rank)
    return [torch.randn(100 + 31 * rank, generator=gen), torch.randn(7, 5, generator=gen) * (1 + rank)]


def _worker(rank, world, port, out_dir):
    os.environ["MASTER_ADDR"] = "127.0.0.1"
    os.environ["MASTER_PORT"] = str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from paper_2101_06983_b200 import sharded
    got = {}
    for name, bound in (("over", 1.0), ("under", 1e6), ("bad", 1.0)):
        grads, st = _parts(rank), torch.zeros(1, dtype=torch.int32)
        if name == "bad" and rank == 1:
            grads[0][3] = math.inf
        sq = sharded.clip_over_ranks(grads, bound, torch.zeros(1, dtype=torch.float64), dev_status=st,
                                     kernels=PlainKernels())
        got[name] = (grads, sq.clone(), st)
    torch.save(got, os.path.join(out_dir, f"r{rank}.pt"))
    dist.barrier()
    dist.destroy_process_group()


@pytest.mark.timeout(180)
def test_two_ranks_clip_by_the_norm_of_both(tmp_path):
    world, port = 2, 30700 + os.getpid() % 1000
    mp.spawn(_worker, args=(world, port, str(tmp_path)), nprocs=world, join=True)
    r = [torch.load(tmp_path / f"r{k}.pt") for k in range(world)]
    whole = [_parts(k) for k in range(world)]
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for p in whole for g in p))
    for k in range(world):
        for name, factor in (("over", 1.0 / (total + 1e-6)), ("under", 1.0)):
            grads, sq, st = r[k][name]
            assert abs(math.sqrt(sq.item()) - total) <= 1e-12 * total and st.item() == 0
            for g, w in zip(grads, whole[k]):
                torch.testing.assert_close(g, w * factor, rtol=2e-7, atol=0)
        grads, sq, st = r[k]["bad"]
        assert not math.isfinite(sq.item()) and st.item() == 8            # on the rank that holds it and on the other
        assert torch.equal(grads[1], whole[k][1])


def test_one_rank_needs_no_group():
    from paper_2101_06983_b200 import sharded
    grads, sq = [torch.full((4,), 2.0)], torch.zeros(1, dtype=torch.float64)
    sharded.clip_over_ranks(grads, 1.0, sq, dev_status=torch.zeros(1, dtype=torch.int32), kernels=PlainKernels())
    assert sq.item() == 16.0
    torch.testing.assert_close(grads[0], torch.full((4,), 0.5), rtol=1e-6, atol=0)


def test_gradients_that_can_be_gone_through_once():
    """(p.grad for p in parameters): read by both passes."""
    from paper_2101_06983_b200 import sharded
    grads, sq = [torch.full((4,), 2.0), torch.full((2, 3), -1.0)], torch.zeros(1, dtype=torch.float64)
    sharded.clip_over_ranks((g for g in grads), 1.0, sq, dev_status=torch.zeros(1, dtype=torch.int32), kernels=PlainKernels())
    assert sq.item() == 22.0
    for g, v in zip(grads, (2.0, -1.0)):
        torch.testing.assert_close(g, torch.full_like(g, v / math.sqrt(22.0)), rtol=1e-6, atol=0)
