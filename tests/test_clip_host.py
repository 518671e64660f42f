"""Gradient clipping, without a GPU: argument checks of the C entry points and of the binding, and the
exchange step of sharded gradients over two gloo ranks."""

import ctypes
import os
from datetime import timedelta

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2609_33645_b200 import binding, data_parallel

BASE = 1 << 20          # made-up addresses: these calls return before they touch a device


def _arr(ctype, values):
    return (ctype * len(values))(*values)


def _call(lib, ptrs, numels, dtypes, outs=None, out_dtypes=None, max_norm=1.0, eps=1e-6, norm=BASE * 32, ws=BASE * 64,
          ws_bytes=1 << 20, n=None):
    return lib.pctc_clip_grad_norm(
        len(ptrs) if n is None else n, _arr(ctypes.c_void_p, ptrs), None if outs is None else _arr(ctypes.c_void_p, outs),
        _arr(ctypes.c_int64, numels), _arr(ctypes.c_int32, dtypes),
        None if out_dtypes is None else _arr(ctypes.c_int32, out_dtypes), max_norm, eps, norm, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(ptrs=[BASE], numels=[-1], dtypes=[0]), 1),
    (dict(ptrs=[None], numels=[8], dtypes=[0]), 1),
    (dict(ptrs=[BASE + 1], numels=[8], dtypes=[0]), 1),                     # not element-aligned
    (dict(ptrs=[BASE + 2], numels=[8], dtypes=[1]), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[2]), 3),
    (dict(ptrs=[BASE], numels=[8], dtypes=[1], outs=[BASE * 2], out_dtypes=[0]), 3),   # fp32 into bf16
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], outs=[BASE], out_dtypes=[1]), 1),       # in place needs one type
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], outs=[None]), 1),
    (dict(ptrs=[BASE, BASE], numels=[8, 8], dtypes=[0, 0]), 1),             # the same tensor twice, in place
    (dict(ptrs=[BASE, BASE + 14], numels=[8, 8], dtypes=[0, 0]), 1),        # one value shared
    (dict(ptrs=[BASE + 16, BASE], numels=[8, 9], dtypes=[0, 0]), 1),        # the same, in falling order
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], outs=[BASE + 8]), 1),        # into itself, shifted
    (dict(ptrs=[BASE, BASE + 64], numels=[8, 8], dtypes=[0, 0], outs=[BASE * 2, BASE]), 1),   # into another's input
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], max_norm=0.0), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], max_norm=-1.0), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], max_norm=float("nan")), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], eps=-1.0), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], eps=float("inf")), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], norm=None), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], ws=None), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], ws=BASE + 8), 1),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], ws_bytes=16), 2),
    (dict(ptrs=[BASE], numels=[8], dtypes=[0], n=-1), 1),
])
def test_bad_lists_are_refused_before_any_launch(lib, kw, want):
    assert _call(lib.load(), **kw) == want


@pytest.mark.parametrize("kw", [
    dict(ptrs=[BASE * 2], numels=[8], dtypes=[1], norm=BASE * 2 + 28),       # the norm on a gradient's last value
    dict(ptrs=[BASE * 2], numels=[8], dtypes=[0], norm=BASE, ws=BASE * 2),   # the workspace on a gradient
    dict(ptrs=[BASE * 2], numels=[8], dtypes=[0], outs=[BASE * 64 + 512]),   # an output in the workspace
    dict(ptrs=[BASE * 2], numels=[8], dtypes=[0], norm=BASE * 64 + 8),       # the norm in the workspace
])
def test_norm_and_workspace_lie_apart_from_the_list(lib, kw):
    assert _call(lib.load(), **kw) == 1


def test_sum_of_squares_lies_apart_from_the_list(lib):
    f, n = lib.load(), _arr(ctypes.c_int64, [8])
    grads, kinds = _arr(ctypes.c_void_p, [BASE * 2]), _arr(ctypes.c_int32, [1])
    assert f.pctc_grad_sqsum(1, grads, n, kinds, BASE * 2 + 24, BASE * 64, 1 << 20, None) == 1
    assert f.pctc_grad_sqsum(1, grads, n, kinds, BASE, BASE * 2, 1 << 20, None) == 1
    assert f.pctc_grad_scale(1, grads, None, n, kinds, None, BASE * 2 + 8, 1.0, 1e-6, BASE, None) == 1
    assert f.pctc_grad_scale(1, grads, None, n, kinds, None, BASE, 1.0, 1e-6, BASE * 2, None) == 1


def test_norm_workspace_and_sum_lie_apart_without_any_tensor(lib):
    f = lib.load()
    assert _call(f, [], [], [], norm=BASE * 64 + 8) == 1
    assert f.pctc_grad_scale(0, None, None, None, None, None, BASE, 1.0, 1e-6, BASE + 4, None) == 1
    assert f.pctc_grad_sqsum(0, None, None, None, BASE * 64 + 16, BASE * 64, 1 << 20, None) == 1


def test_a_misaligned_norm_is_refused(lib):
    for off in (1, 2, 3):
        assert _call(lib.load(), [BASE], [8], [0], norm=BASE * 32 + off) == 1
        f = lib.load().pctc_grad_scale
        assert f(1, _arr(ctypes.c_void_p, [BASE]), None, _arr(ctypes.c_int64, [8]), _arr(ctypes.c_int32, [1]), None, BASE * 2, 1.0,
                 1e-6, BASE * 32 + off, None) == 1


def test_workspace_grows_by_launches_of_1024_tensors(lib):
    a, b, c = (lib.clip_workspace_bytes(n) for n in (1, 1024, 1025))
    assert a == b and a < c < 2 * a + 256


def test_binding_refuses_what_it_cannot_hand_on(lib):
    cpu = torch.zeros(4)
    with pytest.raises(ValueError, match="at least one"):
        binding.clip_grad_norm([], 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        binding.clip_grad_norm([cpu], 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        binding.grad_sqsum([cpu])


def _rank(rank, port, queue):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE="2")
    dist.init_process_group("gloo")
    # the kernels' part replaced by its definition: what is tested is what the ranks exchange
    binding.grad_sqsum = lambda g: dict(sqsum=sum(t.double().square().sum() for t in g).reshape(1))

    def scale(g, sq, max_norm, out=None, eps=1e-6):
        norm = sq.sqrt()
        for t in g:
            t.mul_(torch.clamp(max_norm / (norm + eps), max=1.0).float())
        return dict(norm=norm.float(), grads=g)

    binding.grad_scale = scale
    whole = torch.arange(1, 13, dtype=torch.float32)
    mine = [whole[:5].clone()] if rank == 0 else [whole[5:9].clone(), whole[9:].clone()]
    r = data_parallel.clip_grad_norm_data_parallel(mine, 2.0, sharded=True)
    queue.put((rank, float(r["norm"]), torch.cat(r["grads"]).numpy()))
    dist.barrier()
    dist.destroy_process_group()


def test_sharded_ranks_agree_on_the_norm_of_the_whole():
    ctx = mp.get_context("spawn")
    queue = ctx.Queue()
    port = 29000 + os.getpid() % 1000
    ranks = [ctx.Process(target=_rank, args=(r, port, queue)) for r in range(2)]
    for p in ranks:
        p.start()
    got = sorted((queue.get(timeout=120) for _ in ranks), key=lambda e: e[0])
    for p in ranks:
        p.join(60)
    whole = torch.arange(1, 13, dtype=torch.float64)
    norm = float(whole.norm())
    want = whole * (2.0 / (norm + 1e-6))
    assert got[0][1] == got[1][1] == pytest.approx(norm, rel=2.0 ** -23)
    parts = torch.cat([torch.from_numpy(g[2]) for g in got]).double()
    # the factor and the product each round once to fp32
    assert float(((parts - want).abs() / want).max()) <= 3 * 2.0 ** -24


def _rank_without_a_shard(rank, port, queue):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE="2")
    dist.init_process_group("gloo", timeout=timedelta(seconds=20))
    given = binding.grad_sqsum
    binding.grad_sqsum = lambda g: dict(sqsum=sum(t.double().square().sum() for t in g).reshape(1)) if g else given(g)
    binding.grad_scale = lambda g, sq, max_norm, out=None, eps=1e-6: dict(norm=sq.sqrt().float(), grads=g)
    mine = [torch.full((4,), 3.0)] if rank == 0 else []
    try:
        r = data_parallel.clip_grad_norm_data_parallel(iter(mine), 2.0, sharded=True)
        queue.put((rank, float(r["norm"]), len(r["grads"])))
    except Exception as e:
        queue.put((rank, repr(e), -1))
    dist.destroy_process_group()


def test_a_rank_without_a_shard_takes_its_part():
    ctx = mp.get_context("spawn")
    queue = ctx.Queue()
    port = 30000 + os.getpid() % 1000
    ranks = [ctx.Process(target=_rank_without_a_shard, args=(r, port, queue)) for r in range(2)]
    for p in ranks:
        p.start()
    got = sorted((queue.get(timeout=120) for _ in ranks), key=lambda e: e[0])
    for p in ranks:
        p.join(60)
    assert got == [(0, 6.0, 1), (1, 6.0, 0)]
