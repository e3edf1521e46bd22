"""Steps of AdamW so large that a workgroup takes four stretches of 2048 elements, against the same elements in calls of one stretch a workgroup.

An element's step depends on its own values, its group's and its place, not on who takes it: the bits are the same.  The calls of one stretch are held to the
definition elsewhere, and here at the large call's ends.
"""
import pytest
import torch

from paper_1804_02941_amd import binding as dab
from test_gpu_adamw import check, snapshot

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MANY = 16384 * 2048                    # elements of more stretches than this are taken four at a time


def tensors(n, dtype, bits, seed, copy):
    g = torch.Generator(device=DEV).manual_seed(seed)
    it = {"P": torch.randn(n, generator=g, device=DEV), "G": (0.01 * torch.randn(n, generator=g, device=DEV)).to(dtype), "weight_decay": 0.1,
          "copy": torch.zeros(n, dtype=copy, device=DEV) if copy else None}
    m, root = 0.01 * torch.randn(n, generator=g, device=DEV), 0.01 * torch.rand(n, generator=g, device=DEV)
    it["M"], it["V"] = (dab.dab_state8_save(m, True), dab.dab_state8_save(root, False)) if bits == 8 else (m, root * root)
    return it


def flat(it):
    """All that a step changes, one after the other."""
    return [t for k in ("P", "copy", "M", "V") if it[k] is not None for t in (it[k] if isinstance(it[k], tuple) else (it[k],))]


def cut(it, a, b, place):
    """Elements a .. b - 1 of a tensor, copied; a is a multiple of 32."""
    groups = slice(a // 32, -(-b // 32))
    codes = slice(a, 32 * groups.stop)
    part = {k: tuple(t[s].clone() for t, s in zip(it[k], (codes, groups))) if isinstance(it[k], tuple) else it[k][a:b].clone()
            for k in ("P", "G", "M", "V", "copy") if it[k] is not None}
    return {**part, "copy": part.get("copy"), "weight_decay": it["weight_decay"], "place": place + a}


@pytest.mark.parametrize("bits,dtype,copy", [(8, torch.bfloat16, torch.bfloat16), (32, torch.float32, None), (32, torch.float16, torch.float16)])
def test_four_stretches(bits, dtype, copy):
    n = MANY + 5 * 2048 + 13                                        # the last workgroup's second stretch ends inside a group
    sizes = [100, n, 2049, 33]                                      # workgroups of other tensors before and behind
    items = [tensors(size, dtype, bits, i, copy if i != 2 else None) for i, size in enumerate(sizes)]
    jobs = dab.adamw_jobs(items)
    assert jobs.plan.turns == 4 and jobs.plan.workgroups == sum(-(-size // 8192) for size in sizes)
    parts, place = [], 0
    for it, size in zip(items, sizes):
        edges = [0, 2048 * 5000 + 32, 2 * 8192 * 1000, size] if size == n else [0, size]
        edges.sort()
        parts.append([cut(it, a, b, place) for a, b in zip(edges, edges[1:])])
        place += 32 * -(-size // 32)
    calls = [dab.adamw_jobs([part]) for one in parts for part in one]
    assert all(call.plan.turns == 1 for call in calls)
    first = 128                                                     # the large tensor's place
    ends = [(a, a + many) for a, many in ((0, 64), (8192 * 700 + 2048 * 3, 64), (n // 32 * 32 - 64, 77))]
    before = [snapshot(cut(items[1], a, b, first)) for a, b in ends]
    for step in (1, 2):
        dab.dab_adamw(jobs, 1e-2, step, seed=77)
        for call in calls:
            dab.dab_adamw(call, 1e-2, step, seed=77)
        if step == 1:
            for old, (a, b) in zip(before, ends):
                check(old, cut(items[1], a, b, first), first + a, 1e-2, 1, 0.9, 0.999, 1e-8, 1.0, 77)
    for it, one in zip(items, parts):
        for k, whole in enumerate(flat(it)):
            assert torch.equal(whole, torch.cat([flat(part)[k] for part in one])), k
