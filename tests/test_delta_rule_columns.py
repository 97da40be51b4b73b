"""The gated delta rule where a head's values do not fill the blocks of columns that the kernels take: whatever lies beside a head belongs to another one, or to nobody."""
import pytest
import torch

import seq_util as U
from paper_2305_16513_amd import binding as B
from test_delta_rule import FORWARD, GRADIENT, NAMES, _check, _grads, inputs

gpu = pytest.mark.gpu


# Multiples of 16 that are none of 32, keys of whole tiles, aligned rows, too few states for two columns' groups a workgroup
@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("b,t,hk,hv,dk,dv", [(1, 130, 1, 2, 64, 48), (2, 70, 2, 2, 128, 80), (1, 65, 1, 1, 64, 16), (1, 100, 1, 3, 128, 112), (2, 64, 1, 2, 64, 176)])
def test_values_that_half_fill_the_last_block(dtype, b, t, hk, hv, dk, dv):
    gen = torch.Generator().manual_seed(dv)
    dt = U.TYPES[dtype]
    for gates in (None, torch.float32):
        ins = inputs(gen, b, t, hk, hv, dk, dv, dt, gates)
        go, before, glast = U.normal(gen, b, t, hv, dv, dtype=dt), U.normal(gen, b, hv, dk, dv, std=0.3), U.normal(gen, b, hv, dk, dv)
        gpu_ins = [x.cuda() for x in ins]
        state = before.clone().cuda()
        o = B.sws_delta_rule(*gpu_ins, 0.25, state=state)
        ro, rs = U.delta_rule(*[U.wide(x) for x in ins], 0.25, U.wide(before))
        U.check(o, ro, "o", FORWARD[dtype])
        U.check(state, rs, "state", FORWARD[dtype])
        want = _grads(ins, go, 0.25, before, glast)
        got = B.sws_delta_rule_grad(*gpu_ins, go.cuda(), 0.25, state=before.cuda(), gstate=glast.clone().cuda())
        _check(got, want, ins[0], " with states", dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(64, 16), (64, 48), (128, 80), (100, 40)])
def test_nothing_beside_a_head_is_taken(dtype, dk, dv):
    """Heads of values and of their gradients in wider rows, NaN between them."""
    gen = torch.Generator().manual_seed(dk + dv)
    dt = U.TYPES[dtype]
    b, t, hv = 2, 90, 2
    ins = inputs(gen, b, t, 1, hv, dk, dv, dt)
    go = U.normal(gen, b, t, hv, dv, dtype=dt)

    def apart(x):
        row = torch.full((b, t, hv, dv + 32), float("nan"), dtype=dt, device="cuda")
        row[..., :dv] = x.cuda()
        return row[..., :dv]
    gpu_ins = [x.cuda() for x in ins]
    gpu_ins[2] = apart(ins[2])
    ro, rs = U.delta_rule(*[U.wide(x) for x in ins], 0.25)
    state = torch.zeros(b, hv, dk, dv, device="cuda")
    U.check(B.sws_delta_rule(*gpu_ins, 0.25, state=state), ro, "o", FORWARD[dtype])
    U.check(state, rs, "state", FORWARD[dtype])
    glast = U.normal(gen, b, hv, dk, dv)
    want = _grads(ins, go, 0.25, torch.zeros(b, hv, dk, dv), glast)
    got = B.sws_delta_rule_grad(*gpu_ins, apart(go), 0.25, gstate=glast.clone().cuda())
    for x, r, name in zip(got, want, NAMES):
        U.check(x, r, name, GRADIENT[dtype])
