"""Data errors of the experts' calls reach a caller who passes an `err` tensor, through all the calls that share it; the example does."""
import pytest
import torch

import paper_2606_01007_amd as tacg
from test_gpu_moe_layer import ROOT, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def test_the_example_looks_at_its_errors():
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.run(steps=3, say=lambda *_: None)["err"] == 0


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_one_tensor_collects_the_errors_of_several_calls(mode):
    g = torch.Generator().manual_seed(1)
    w = torch.randn((4, 32, 64), generator=g).cuda()
    x = torch.randn((40, 64), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(0, 4, (40, 2), generator=g).to(torch.int16)
    gate = torch.ones((40, 2), device="cuda") if mode == "sum" else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, s, _ = tacg.q4_pack(w, group=32, err=err)
    call = lambda i: tacg.expert_q4(x, i.cuda(), q, s, group=32, mode=mode, gate=gate, err=err)  # noqa: E731
    call(ids)
    assert int(err.item()) == 0
    w[0, 0, 0] = float("inf")
    tacg.q4_pack(w, group=32, err=err)
    assert int(err.item()) == tacg.ERR_VALUE
    ids[39, 1] = 4
    call(ids)
    assert int(err.item()) == tacg.ERR_VALUE | tacg.ERR_ID_RANGE
