"""The fp32 outputs of the gated delta rule on 16-bit storage (states, gradients of states and of fp32 gates) against 64 bits: they are as exact as fp32 products leave
them, whether a call's tokens are few or many."""
import pytest
import torch

import seq_util as U
from paper_2305_16513_amd import binding as B
from test_delta_rule import _grads, inputs

gpu = pytest.mark.gpu

# Root mean squares of the error, relative to that of the result.  Some eight products in a row, in each of which a sum is rounded some 32 times by 2^-24 of itself at
# most: sqrt(8 * 32) * 2^-24 = 1e-6.  A gradient of a gate is a sum of differences of larger terms: four times that.  (One piece less of a bf16 operand, off by 2^-17, shows as 3e-6
# to 5e-6 and 5e-6 to 1e-5.)
EXACT = {"state": 1e-6, "gstate": 1e-6, "gbeta": 1e-6, "gg": 4e-6}


def off(got, ref):
    ref = ref.detach()
    return ((got.double().cpu() - ref).square().mean().sqrt() / ref.square().mean().sqrt()).item()


def calls(gen, dtype, b, t, hk, hv, dk, dv, go_size=1.0, v_size=1.0, state_size=0.3, mild=False):
    """What a call and its gradients give in fp32, and the same in 64 bits."""
    ins = list(inputs(gen, b, t, hk, hv, dk, dv, U.TYPES[dtype], torch.float32))
    ins[2] = (ins[2].float() * v_size).to(ins[2].dtype)
    if mild:
        ins[3] = ins[3] / 32
    go = (U.normal(gen, b, t, hv, dv) * go_size).to(U.TYPES[dtype])
    before, glast = U.normal(gen, b, hv, dk, dv) * state_size, U.normal(gen, b, hv, dk, dv) * go_size
    state = before.clone().cuda()
    gpu_ins = [x.cuda() for x in ins]
    o = B.sws_delta_rule(*gpu_ins, 0.25, state=state)
    got = B.sws_delta_rule_grad(*gpu_ins, go.cuda(), 0.25, state=before.cuda(), gstate=glast.clone().cuda())
    ro, rs = U.delta_rule(*[U.wide(x) for x in ins], 0.25, U.wide(before))
    want = _grads(ins, go, 0.25, before, glast)
    names = ("gq", "gk", "gv", "gg", "gbeta", "gstate")
    return {"o": o, "state": state, **dict(zip(names, got))}, {"o": ro, "state": rs, **dict(zip(names, want))}


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("t,hv,dk,dv,mild", [(300, 2, 128, 128, False), (300, 1, 128, 64, True), (200, 2, 64, 64, False), (140, 1, 100, 36, False)])
def test_fp32_outputs_are_exact_to_fp32(dtype, t, hv, dk, dv, mild):
    got, want = calls(torch.Generator().manual_seed(t + dk), dtype, 1, t, 1, hv, dk, dv, mild=mild)
    for name, bound in EXACT.items():
        assert off(got[name], want[name]) <= bound, (name, off(got[name], want[name]))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_state_does_not_depend_on_how_many_tokens_a_call_has(dtype):
    """A prompt in one call and the same tokens in calls of a few."""
    gen = torch.Generator().manual_seed(9)
    ins = [x.cuda() for x in inputs(gen, 1, 192, 1, 2, 128, 128, U.TYPES[dtype], torch.float32)]
    whole, pieces = (torch.zeros(1, 2, 128, 128, device="cuda") for _ in range(2))
    B.sws_delta_rule(*ins, 0.25, state=whole)
    for t in range(0, 192, 8):
        B.sws_delta_rule(*[x[:, t:t + 8] for x in ins], 0.25, state=pieces)
    assert off(whole, pieces.double().cpu()) <= EXACT["state"]


# Gradients of a loss that is a mean over tokens, small values and states, states beyond what fp16 holds (which single tokens take too); of these, little is forgotten: fp16's
# pieces hold 2^-25 of the largest number, not of what is left of it
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("go_size,v_size,state_size", [(1e-4, 1, 0.3), (1e-6, 1, 0.3), (1, 1e-3, 1e-3), (1, 1, 1e5), (100, 3000, 1e6), (1e-5, 1e-4, 1e-7)])
@pytest.mark.parametrize("hv,dk,dv", [(2, 128, 64), (1, 64, 128), (3, 40, 50)])
def test_sizes_far_from_one(dtype, go_size, v_size, state_size, hv, dk, dv):
    got, want = calls(torch.Generator().manual_seed(dk + dv), dtype, 2, 150, 1, hv, dk, dv, go_size, v_size, state_size, mild=state_size > 1)
    for name, bound in EXACT.items():
        assert off(got[name], want[name]) <= bound, (name, off(got[name], want[name]))
    # outputs of 16 bits: their own rounding, of a fixed size below fp16's normal numbers
    for name in ("o", "gq", "gk", "gv"):
        x, r = got[name].double().cpu(), want[name].detach()
        fits = r.abs() < 60000
        allowed = U.HALF[got[name].dtype] * r.abs() * (1 + 2.0 ** -6) + 2e-5 * r.square().mean().sqrt() + (2.0 ** -25 if dtype == "f16" else 0)
        assert bool(((x - r).abs() <= allowed)[fits].all()), name


@gpu
@pytest.mark.parametrize("b,t", [(1, 8), (1, 9), (16, 15), (16, 16), (128, 48), (128, 49)])
def test_states_on_both_sides_of_what_few_tokens_are(b, t):
    """How many tokens are taken one by one depends on the number of states; a state's precision does not."""
    got, want = calls(torch.Generator().manual_seed(b + t), "bf16", b, t, 16, 16, 20, 24)
    assert off(got["state"], want["state"]) <= EXACT["state"]
