"""attention(qk_norm, rope) writes to the caller's Q and K before its other calls run: whatever any of the calls refuses is
refused while Q and K are as they were."""
import dataclasses

import pytest
import torch

from gpu_harness import SMALL, inputs, problem_of, to_device
from paper_2609_32628_amd import _lib, api

pytestmark = pytest.mark.gpu


def small(t):
    return t.flatten()[:16]


def strided(t):
    """The same values, with gaps between the heads' rows."""
    room = torch.empty(t.shape[:3] + (2 * t.shape[3],), dtype=t.dtype, device=t.device)
    room[..., :t.shape[3]] = t
    return room[..., :t.shape[3]]


CHANGES = {
    "w_q of another width": lambda a: a.update(qk_norm=(torch.ones(64, device="cuda"), None)),
    "w_k of another width": lambda a: a.update(qk_norm=(None, torch.ones(64, device="cuda"))),
    "w_k of another type": lambda a: a.update(qk_norm=(None, torch.ones(128, device="cuda", dtype=torch.float64))),
    "w_k on the CPU": lambda a: a.update(qk_norm=(None, torch.ones(128))),
    "K of other strides": lambda a: a.update(K=strided(a["K"])),
    "K of another type": lambda a: a.update(K=a["K"].float()),
    "K of fewer tokens": lambda a: a.update(K=a["K"][:, :, :-1].contiguous()),
    "V of other strides": lambda a: a.update(V=strided(a["V"])),
    "V of another type": lambda a: a.update(V=a["V"].float()),
    "V in K's memory": lambda a: a.update(V=a["K"]),
    "V in Q's memory": lambda a: a.update(V=a["Q"]),
    "O of another shape": lambda a: a.update(O=a["O"][:, :, :-1]),
    "O of rows that repeat": lambda a: a.update(O=a["O"][:, :1].expand_as(a["O"])),
    "O in half precision": lambda a: a.update(O=a["O"].half()),
    "Q, K and V in half precision": lambda a: a.update({n: a[n].half() for n in "QKV"}),
    "a lambda above 1": lambda a: a.update(lam=1.5),
    "budgets above the whole": lambda a: a.update(budgets=(60, 60, 100)),
    "budgets of two numbers": lambda a: a.update(budgets=(10, 30)),
    "a 16-bit budget without its buffers": lambda a: a.update(num16=1),
    "a rope block that does not divide the head": lambda a: a.update(rope=api.da2_rope_plan(96, (96,))),
    "a rope of two axes": lambda a: a.update(rope=api.da2_rope_plan(128, (64, 64))),
    "a rope of odd channels": lambda a: a.update(rope=api.Rope("half", 128, (63,), torch.zeros(31, dtype=torch.float64, device="cuda"))),
    "a rope beyond its block": lambda a: a.update(rope=api.Rope("half", 64, (128,), torch.zeros(64, dtype=torch.float64, device="cuda"))),
    "a rope of an unknown layout": lambda a: a.update(rope=api.Rope("other", 128, (128,), torch.zeros(64, dtype=torch.float64, device="cuda"))),
    "a rope with too few turns": lambda a: a.update(rope=dataclasses.replace(a["rope"], turns=a["rope"].turns[:-1])),
    "turns on the CPU": lambda a: a.update(rope=dataclasses.replace(a["rope"], turns=a["rope"].turns.cpu())),
    "a rope of no finite scale": lambda a: a.update(rope=dataclasses.replace(a["rope"], scale=float("nan"))),
    "a short operand buffer": lambda a: a.update(buf=dataclasses.replace(a["buf"], ops=small(a["buf"].ops))),
    "a short draft workspace": lambda a: a.update(buf=dataclasses.replace(a["buf"], ws_draft=small(a["buf"].ws_draft))),
    "a short ranking workspace": lambda a: a.update(buf=dataclasses.replace(a["buf"], ws_rank=small(a["buf"].ws_rank))),
    "the lists of a smaller problem": lambda a: a.update(buf=dataclasses.replace(a["buf"], lists=small(a["buf"].lists))),
    "a problem of fewer tokens": lambda a: a.update(buf=dataclasses.replace(a["buf"], p=api.problem(SMALL.B, SMALL.H, SMALL.d, SMALL.T, 13, 20))),
}


def arguments():
    Q, K, V = (to_device(x, SMALL) for x in inputs(SMALL))
    return dict(Q=Q, K=K, V=V, buf=api.alloc(problem_of(SMALL), SMALL.scope), lam=SMALL.lam, budgets=SMALL.budgets, O=torch.empty_like(Q),
                num16=0, qk_norm=(torch.full((128,), 0.5, device="cuda"), None), rope=api.da2_rope_plan(128, (44, 42, 42)))


@pytest.mark.parametrize("name", CHANGES)
def test_a_refused_call_leaves_q_and_k(name):
    a = arguments()
    CHANGES[name](a)
    before = a["Q"].clone(), a["K"].clone()
    with pytest.raises((ValueError, KeyError, TypeError, _lib.Da2Error)):
        api.attention(**a)
    torch.cuda.synchronize()
    assert torch.equal(a["Q"], before[0]) and torch.equal(a["K"], before[1])


def test_the_call_itself_is_taken():
    for fmt4, with16, num16 in (("nvfp4", False, 0), ("mxfp4", False, 0), ("nvfp4", True, 5)):
        a = arguments()
        a.update(buf=api.alloc(problem_of(SMALL), SMALL.scope, fmt4=fmt4, with16=with16), num16=num16)
        assert api.attention(**a).isfinite().all()
