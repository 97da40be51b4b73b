"""The gated delta rule where numbers are not finite."""
import pytest
import torch

import seq_util as U
from paper_2305_16513_amd import binding as B
from test_delta_rule import FORWARD, inputs

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv,t", [(64, 64, 150), (100, 36, 150), (128, 128, 90), (64, 64, 6)])
def test_tokens_that_are_not_there_have_zeros_whatever_the_state(dtype, dk, dv, t):
    gen = torch.Generator().manual_seed(dk + t)
    n = torch.tensor([t, t - 5, 3, 0, 70], dtype=torch.int32)
    b = len(n)
    ins = [x.cuda() for x in inputs(gen, b, t, 1, 2, dk, dv, U.TYPES[dtype])]
    go = U.normal(gen, b, t, 2, dv, dtype=U.TYPES[dtype]).cuda()
    for bad in (float("nan"), float("inf")):
        before, glast = (torch.full((b, 2, dk, dv), bad, device="cuda") for _ in range(2))
        o = B.sws_delta_rule(*ins, 0.25, state=before.clone(), lengths=n.cuda())
        got = B.sws_delta_rule_grad(*ins, go, 0.25, state=before, gstate=glast, lengths=n.cuda())
        for x, name in zip((o,) + tuple(got[:5]), ("o", "gq", "gk", "gv", "gg", "gbeta")):
            for i in range(b):
                assert not bool((x[i, min(int(n[i]), t):] != 0).any()), (name, i)
        for i in range(b):
            assert not torch.isfinite(o[i, :min(int(n[i]), t)]).any(), i


def _finite_part(ins, scale, before):
    """o and the last state in 64 bits, as far as they are finite; what is not, is not finite in the result either."""
    return U.delta_rule(*[U.wide(x) for x in ins], scale, U.wide(before))


# Places in a chunk: its first token, inside and between tiles of 16, its halves, its last; in the first chunk and behind it; in a chunk that is filled in part
@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 48), (40, 36)])
@pytest.mark.parametrize("at", [0, 5, 16, 31, 32, 40, 63, 64, 90, 127, 128, 133])
def test_what_is_not_finite_reaches_no_earlier_token(dtype, dk, dv, at):
    """A token's key, value, gate or learning rate that is not finite: outputs before it are as without it.  A value's element stays in its column, a query's in its token."""
    gen = torch.Generator().manual_seed(dk + at)
    dt, t, hv = U.TYPES[dtype], 140, 2
    for bad in (float("nan"), float("inf")):
        for which, name in enumerate(("q", "k", "v", "g", "beta")):
            if name == "g" and bad > 0:
                continue                                     # (gates are at most 0)
            ins = list(inputs(gen, 1, t, 1, hv, dk, dv, dt))
            before = U.normal(gen, 1, hv, dk, dv, std=0.3)
            ref = [x.clone() for x in ins]
            if name == "v":
                ins[2][0, at, 0, 3] = bad
            elif name in ("q", "k"):
                ins[which][0, at, 0, 3] = bad
            else:
                ins[which][0, at, 0] = bad
            state = before.clone().cuda()
            o = B.sws_delta_rule(*[x.cuda() for x in ins], 0.25, state=state)[0].cpu()
            ro, rs = _finite_part(ref, 0.25, before)
            ro, rs, last = ro[0], rs[0], state[0].cpu()
            U.check(o[:at], ro[:at], name, FORWARD[dtype])
            if name == "q":                                  # (both heads read it)
                assert not torch.isfinite(o[at]).any()
                U.check(o[at + 1:], ro[at + 1:], name, FORWARD[dtype])
                U.check(last, rs, "state", FORWARD[dtype])
            elif name == "v":
                others = [d for d in range(dv) if d != 3]
                assert not torch.isfinite(o[at:, 0, 3]).any() and not torch.isfinite(last[0, :, 3]).any()
                U.check(o[:, 0, others], ro[:, 0, others], name, FORWARD[dtype])
                U.check(last[0][:, others], rs[0][:, others], "state", FORWARD[dtype])
            else:
                assert not torch.isfinite(o[at:, 0]).any() and not torch.isfinite(last[0]).any()
            if name != "k" and name != "q":
                U.check(o[:, 1], ro[:, 1], "the other head", FORWARD[dtype])
                U.check(last[1], rs[1], "the other head's state", FORWARD[dtype])


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_several_tokens_that_are_not_finite(dtype):
    gen = torch.Generator().manual_seed(7)
    ins = list(inputs(gen, 1, 100, 1, 1, 64, 64, U.TYPES[dtype]))
    ref = [x.clone() for x in ins]
    places = {0: 70, 1: 3, 7: 64, 20: 50, 33: 17, 63: 99}    # column: its first such token
    for c, t in places.items():
        ins[2][0, t, 0, c] = float("inf")
        ins[2][0, min(t + 9, 99), 0, c] = float("nan")
    ins[0][0, 10, 0, 0] = float("nan")
    ins[0][0, 80, 0, 5] = float("inf")
    state = torch.zeros(1, 1, 64, 64, device="cuda")
    o = B.sws_delta_rule(*[x.cuda() for x in ins], 0.25, state=state)[0, :, 0].cpu()
    ro, rs = U.delta_rule(*[U.wide(x) for x in ref], 0.25)
    good = torch.ones(100, 64, dtype=torch.bool)
    for c, t in places.items():
        good[t:, c] = False
    good[[10, 80]] = False
    assert torch.equal(torch.isfinite(o), good)
    U.check(torch.where(good, o, 0), torch.where(good, ro[0, :, 0], 0), "o", FORWARD[dtype])
    columns = [c for c in range(64) if c not in places]
    U.check(state[0, 0][:, columns], rs[0, 0][:, columns], "state", FORWARD[dtype])
