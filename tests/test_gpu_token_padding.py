"""What lies past a sequence's length has no part in a training step of the token model, whatever it holds."""
import pytest
import torch

from gpu_common import check_status
from test_gpu_token_step import TS, setup  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", ["bf16", "f16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -1e4])
@pytest.mark.parametrize("graph", [False, True])
def test_features_past_a_length_do_not_count(TS, prec, value, graph):  # noqa: F811
    outs = []
    for fill in (0.0, value):
        D, spec, server, wk, x = setup(TS, prec)
        wk.set_lengths(torch.tensor([70, 1, 33], dtype=torch.int32))
        for b, ln in enumerate((70, 1, 33)):
            x[b, ln:] = fill
            wk.labels.view(3, 70)[b, ln:] = -5
        it = TS.DualBatchIteration(server, wk, None, wk.res, lr=0.1)
        it.set_inputs(x, wk.labels.clone())
        if graph:
            it.capture()
        it.run()
        check_status(D)
        outs.append([t.clone() for t in (server.w, wk.loss, wk.grad, wk.dfeatures, wk.h_last)])
        assert all(bool(torch.isfinite(t.float()).all()) for t in outs[-1])
        assert not wk.dfeatures.view(x.shape)[1, 1:].any()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
