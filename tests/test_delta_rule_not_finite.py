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
