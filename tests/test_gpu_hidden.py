"""Hidden states of batches that the GEMV path serves in several groups of rows."""
import numpy as np
import pytest

from oracle import gpt as ogpt
from paper_2607_21042_amd import workload
from tests import helpers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [17, 40])
def test_hidden_states_of_every_group(B):
    """fp32 takes at most 16 rows a launch: each launch writes its own rows of hidden_out."""
    from paper_2607_21042_amd import ftts
    shape = workload.TINY
    master = workload.master_weights(shape, seed=0)
    dm = ftts.DeviceModel(master, shape, ftts.F32)
    om = ogpt.GPT(master, shape.n_head, shape.d_head, dtype=np.float32)
    lens = [3 + b % 5 for b in range(B)]
    prefixes = np.split(workload.prefix_embeddings(lens, shape.d_model, seed=1, bf16=False), np.cumsum(lens)[:-1])
    fed = workload.random_tokens(2, B, shape.vocab, seed=6)
    print(f"hidden states: B {B}", flush=True)
    res = helpers.run_gpu(dm, shape, prefixes, fed, hidden=True)
    for b in range(B):
        _, _, ref = helpers.oracle_teacher_forced(om, prefixes[b], fed[:, b], with_hidden=True)
        for t in range(2):
            ok, err = helpers.tolerance_ok(res["hidden"][t, b], ref[t], "f32")
            assert ok, (t, b, err)
