"""HierAvg.scores (the rows behind evaluate) against the oracle's logits of the
same parameters, and against evaluate itself.

The logits come from the forward that evaluate takes, whose loss is held to
1e-4 of the oracle's; a row's log probability, entropy and order move with its
logits: by at most twice (the entropy: twice log C times) their error, which
float32 sums of n products keep below sqrt(n) 2^-22 of the largest logit plus
its terms; 1e-4 of the largest logit covers the widest case here."""

import numpy as np
import pytest

import cases
from oracle import method as M
from oracle import rng
from test_gpu_parity import EVAL_CASES

pytestmark = pytest.mark.gpu


def oracle_logits(p, row, n, split):
    blk = M.unpack(p, row)
    X, y = rng.data_rows(p.seed, np.arange(n), p.IN, p.C, p.sigma, split)
    if p.kind == M.SOFTMAX:
        return X @ blk["W"].T + blk["b"], y
    return np.maximum(X @ blk["W1"].T + blk["b1"], 0.0) @ blk["W2"].T + blk["b2"], y


@pytest.mark.parametrize("name", sorted(EVAL_CASES))
def test_scores_match_the_oracle_and_evaluate(name, gpu_lib):
    from paper_1903_05133_amd import HierAvg
    c, mode = EVAL_CASES[name]
    prob = cases.oracle_problem(c)
    with HierAvg(config=cases.native_config(c, mode)) as h:
        h.round()
        W = h.params().astype(np.float64)
        plan = [(0, 0, min(c["N"], 300)), (c["P"] - 1, 1, 300 if c["IN"] > 1000 else 5000)]
        for replica, split, n in plan:
            top = min(3, c["C"])
            print(f"[gpu case] scores {name} replica {replica} split {split} rows {n}", flush=True)
            logp, ent, ids, tl = h.scores(replica, split, n, top)
            loss, correct = h.evaluate(replica, split, n)
            assert abs(-logp.astype(np.float64).mean() - loss) <= 1e-5 * max(1.0, abs(loss))
            z, y = oracle_logits(prob, W[replica], n, split)
            d = z - z.max(1, keepdims=True)
            logs = d - np.log(np.exp(d).sum(1, keepdims=True))
            tol = 1e-4 * np.maximum(1.0, np.abs(z).max(1))
            rows = np.arange(n)
            assert np.all(np.abs(logp - logs[rows, y]) <= 2 * tol)
            want = -(np.exp(logs) * logs).sum(1)
            assert np.all(np.abs(ent - want) <= 2 * tol * max(1.0, np.log(c["C"])))
            # the classes named hold what is said of them, and none left out is larger by more than rounding
            assert np.all(np.abs(tl - logs[rows[:, None], ids]) <= 2 * tol[:, None])
            assert np.all(np.diff(tl, axis=1) <= 0)
            best = -np.sort(-logs, axis=1)[:, :top]
            assert np.all(np.abs(tl - best) <= 2 * tol[:, None])
            assert abs(int((ids[:, 0] == y).sum()) - correct) <= int(((best[:, 0] - best[:, min(1, top - 1)]) < 1e-5).sum())
        # the same call again, in fewer rows, and into device memory through the C entry
        import torch
        a = h.scores(replica, split, 17, top)
        for x, full in zip(a, (logp, ent, ids, tl)):
            assert np.allclose(x, full[:17], rtol=1e-4, atol=1e-4)
        dev = [torch.empty(x.shape, dtype=torch.int32 if x.dtype == np.int32 else torch.float32, device="cuda") for x in a]
        torch.cuda.synchronize()
        assert gpu_lib.hieravg_scores(h._h, replica, split, 17, top, *(t.data_ptr() for t in dev)) == 0
        for x, t in zip(a, dev):
            assert np.array_equal(x, t.cpu().numpy())
        for bad in ((c["P"], 0, 10, 1), (0, 2, 10, 1), (0, 0, c["N"] + 1, 1), (0, 0, 10, min(c["C"], 64) + 1), (0, 0, 0, 0),
                    (0, 0, 10, -1)):
            with pytest.raises(RuntimeError):
                h.scores(*bad)


def test_scores_of_the_averaging_kind_refused(gpu_lib):
    from paper_1903_05133_amd import HierAvg, config
    with HierAvg(config=config(2, 2, 1, 1, 1, in_dim=64, momentum=0.9)) as h:
        with pytest.raises(RuntimeError, match="no model"):
            h.scores(0, 0, 4, 0)
