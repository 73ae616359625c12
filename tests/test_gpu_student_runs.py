"""A student in two stages (rotary positions, norm joins, norms without a mean, distillation) through what every stage takes: checkpoints of its stages, and the comparison schedule
with a distillation's records as labels."""
import numpy as np
import pytest

from oracle import baseline
from tests.test_gpu_operator_layers import both, student
from tests.util import rel_err

pytestmark = pytest.mark.gpu


@both
def test_resume_from_stage_checkpoints(dtype, tmp_path):
    """Bit for bit as the run that wrote them; parameters, momentum and counter of norms that have no shift among them."""
    from paper_2410_14312_amd import Pipeline

    cfg, params, batches = student(dtype)
    a = Pipeline(cfg, params)
    a.run(batches[:2])
    a.save_checkpoint(str(tmp_path), 1)
    want, _ = a.run(batches[2:])
    b = Pipeline(cfg, params)
    assert b.resume(str(tmp_path)) == 1 and [st.version() for st in b.stages] == [2] * cfg.K
    got, _ = b.run(batches[2:])
    assert got == want
    for s in range(cfg.K):
        for of in (lambda st: st.get_params(), lambda st: st.get_momentum()):
            for p, q in zip(of(a.stages[s]), of(b.stages[s])):
                assert p.keys() == q.keys() and all(np.array_equal(p[k], q[k]) for k in p)
        assert any(set(p) == {"w"} for p in b.get_params(s))


@both
def test_the_comparison_schedule(dtype):
    """1F1B with kept versions: losses and weights as the oracle's (bars of tests/test_gpu_operator_layers.py for the student's own schedule)."""
    from paper_2410_14312_amd import Pipeline

    cfg, params, batches = student(dtype)
    small = [(x[i:i + 2], y[i:i + 2]) for x, y in batches for i in range(0, cfg.M, 2)][:9]
    ref = baseline.run_1f1b(cfg.stages, params, small, cfg.lr, cfg.momentum, precision="bf16" if dtype == "bf16" else "f64")
    pipe = Pipeline(cfg, params, baseline_1f1b=True, batch=2)
    losses, log = pipe.run(small)
    assert np.array_equal(log, np.array(ref["ops"], dtype=np.int32))
    tol = 1e-4 if dtype == "f32" else 4e-2
    assert np.max(np.abs(np.array(losses) - ref["losses"]) / np.abs(ref["losses"])) < tol, (losses, ref["losses"])
    for s in range(cfg.K):
        for got, want in zip(pipe.get_params(s), ref["stages"][s].params):
            for k in want:
                assert rel_err(got[k].reshape(want[k].shape), want[k]) < tol
