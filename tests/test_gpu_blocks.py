"""Rounds of the MLP of residual blocks (abs_create_blocks) against the oracle, its evaluation, batches and repeatability."""
import numpy as np
import pytest
import torch

import workloads
import paper_2301_08895_amd as lib
from oracle import blocks as ob
from oracle.bf16 import bits_to_f64

pytestmark = pytest.mark.gpu

# Between a matrix gradient and the models lie at most seven roundings to bf16, half a step 2^-8 of a value at most; the oracle
# makes the same ones, and a sum that lands on the other side of a rounding point moves a value by one step.
TOL = 7 * 2.0 ** -8


def preset(**over):
    blocks = {k: over.pop(k) for k in ("groups", "act", "residual", "drop") if k in over}
    base = dict(M=3000, dims=[48, 64, 64, 10], N=6, B=20, n_slow=1, lr=0.05, K0=3, k_mode=1, tau_cap=3)
    base.update(over)
    base["n_classes"] = base["dims"][-1]                  # (labels are in [0, d_L))
    p = workloads.scaled_preset(3, **base)
    return workloads.with_blocks(p, **{"groups": 8, "drop": 13107, **blocks})


def tensors(p):
    d, out, o = p["dims"], [], 0
    for l in range(len(d) - 1):
        sizes = ([("gamma", d[l]), ("beta", d[l])] if l else []) + [("W", d[l] * d[l + 1]), ("b", d[l + 1])]
        for name, n in sizes:
            out.append((f"{name}{l}", slice(o, o + n)))
            o += n
    return out


def oracle_rounds(p, d, sim, T):
    """Models w^0 .. w^T and mean losses, following the event trace of the handle."""
    cfg, opt, dims, B = sim.cfg, p["blocks"], p["dims"], p["B"]
    X, y = bits_to_f64(d["X"]), d["y"]
    jobs, models, losses = [0] * p["N"], [d["w0"].astype(np.float64)], []
    for t, rec in enumerate(sim.trace(0, T)):
        K, n_restart = int(rec[1]), int(rec[5])
        ids, vers = rec[12:12 + K], rec[12 + K:12 + 2 * K]
        taus = rec[12 + 2 * K:12 + 3 * K]
        order = sorted(range(K), key=lambda a: vers[a])                    # stable: arrival order inside a version
        masks = [None] + [ob.kept(K * B, dims[l], opt["drop"], p["seed_sim"], 8 * t + l) for l in range(1, len(dims) - 1)]
        w, total, at = models[t].copy(), 0.0, 0
        groups = {}
        for pos, a in enumerate(order):
            groups.setdefault(int(vers[a]), []).append((pos, a))
        for v in sorted(groups):
            rows, coef = [], []
            for pos, a in groups[v]:
                rows += list(lib.abs_draw_batch_rows(cfg, int(ids[a]), jobs[int(ids[a])]))
                eta = p["lr"] / max(1, int(taus[a])) if p["sa_penalty"] else p["lr"]
                coef += [np.float32(eta / (K * B))] * B
            span = slice(groups[v][0][0] * B, (groups[v][-1][0] + 1) * B)
            g, per_row = ob.gradient(dims, opt, models[v], X[rows], y[rows], np.array(coef, dtype=np.float64),
                                     [None] + [m[span] for m in masks[1:]])
            w -= g
            total += per_row.reshape(-1, B).mean(1).sum()
        losses.append(total / K)
        models.append(w)
        for n in set(int(i) for i in ids) | set(int(i) for i in rec[12 + 3 * K:12 + 3 * K + n_restart]):
            jobs[n] += 1
    return models, losses


@pytest.mark.parametrize("over", [dict(), dict(residual=0, act=3, drop=0), dict(act=0, dims=[64, 40, 24, 40, 5], groups=4, sa_penalty=1),
                                  dict(dims=[16, 50, 50, 50, 26], groups=5, B=33, N=9, K0=9, drop=32768),
                                  dict(dims=[200, 128, 3], groups=1, B=1, N=12, K0=5)])
def test_rounds_follow_the_oracle(over):
    p = preset(**over)
    d = workloads.make_inputs(p)
    sim = lib.Simulation(p, d)
    T = 8
    got = [sim.model()]
    for _ in range(T):
        sim.round(1)
        got.append(sim.model())
    want, losses = oracle_rounds(p, d, sim, T)
    trace = sim.trace()
    assert max(int(v) for r in trace for v in r[12 + 2 * int(r[1]):12 + 3 * int(r[1])]) > 0 or p["K0"] == p["N"]     # stale gradients occurred
    for t in range(T):
        gl = float(trace[t][10:11].view(np.float32)[0])
        assert abs(gl - losses[t]) <= TOL * max(1.0, losses[t]), t
    for t in (1, T):
        for name, s in tensors(p):
            up, back = got[t][s].astype(np.float64) - got[0][s], want[t][s] - want[0][s]
            assert np.linalg.norm(up - back) <= TOL * max(np.linalg.norm(back), 1e-12), (t, name)
    sim.close()


def test_evaluation_and_its_static_form():
    p = preset()
    d, Xe, ye = workloads.make_split(p, 777)              # six passes of N B = 120 rows, then 40 + 17
    sim = lib.Simulation(p, d)
    sim.round(5)
    loss, acc = sim.evaluate(Xe, ye)
    z, _ = ob.forward(p["dims"], p["blocks"], sim.model(), bits_to_f64(Xe))
    per_row, _ = ob.loss_of(z, ye)
    top2 = np.sort(z, axis=1)[:, -2:]
    near = (top2[:, 1] - top2[:, 0] <= TOL * np.abs(z).max(1)).mean()
    assert abs(loss - per_row.mean()) <= TOL * max(1.0, per_row.mean())
    assert abs(acc - (z.argmax(1) == ye).mean()) <= near + 1e-12
    xt, yt = torch.from_numpy(Xe.view(np.int16)).cuda(), torch.from_numpy(ye).cuda()
    out = torch.zeros(2, dtype=torch.float64, device="cuda")
    lib.abs_evaluate_static(sim.handle, -1, xt.data_ptr(), yt.data_ptr(), 777, out.data_ptr())
    assert out.tolist() == [loss, acc]
    old = sim.model(4)
    sim.round(1)
    assert np.array_equal(sim.model(4), old)
    sim.close()


def test_runs_and_batches_give_the_same_bits():
    p = preset(k_mode=0)
    d = workloads.make_inputs(p)

    def alone(seed):
        s = lib.Simulation(dict(p, seed_sim=seed), d)
        s.round(6)
        return s

    runs = [alone(3), alone(3), alone(4)]
    assert np.array_equal(runs[0].model(), runs[1].model()) and not np.array_equal(runs[0].model(), runs[2].model())
    sims = [lib.Simulation(dict(p, seed_sim=s), d) for s in (3, 4, 5)]
    batch = lib.Batch(sims)
    batch.round(6)
    assert np.array_equal(sims[0].model(), runs[0].model()) and np.array_equal(sims[1].model(), runs[2].model())
    batch.close()
    plain = {k: v for k, v in p.items() if k != "blocks"}
    other = lib.Simulation(plain, workloads.make_inputs(plain))
    with pytest.raises(lib.AbsError):
        lib.Batch([sims[0], other])                       # one with blocks, one without
    for s in runs + sims + [other]:
        s.close()


def test_operators_are_what_a_round_runs():
    p = preset()
    sim = lib.Simulation(p, workloads.make_inputs(p), profile=1)
    sim.round(3)
    stats = {s["name"]: s for s in sim.kernel_stats()}
    assert {"blocks_linear", "blocks_norm", "blocks_dropout", "blocks_loss", "blocks_update"} <= set(stats)
    assert all(s["total_ms"] > 0 for n, s in stats.items() if n.startswith("blocks"))
    sim.close()


def test_comparison_command(capsys):
    from paper_2301_08895_amd import compare
    assert compare.main(["--config", "3", "--blocks", "16", "--dropout", "0.2", "--methods", "abs,k_async", "--rounds", "4", "--every", "2",
                         "--M", "2000", "--eval-rows", "300"]) == 0
    assert "k_async" in capsys.readouterr().out
