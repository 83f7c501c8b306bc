"""Host-side checks of libabs that need no GPU: the library loads and exports every
symbol include/abs.h declares, the config mirror matches, and the host scheduler
(schedule-only mode) reproduces the oracle's integer event trace bit for bit."""
import ctypes
import os
import re

import numpy as np
import pytest

import workloads
import paper_2301_08895_amd as lib
from oracle import counter_rng as crng
from oracle.abs_sim import AbsOracle, trace_words
from parity_util import hand_worked_schedule

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported():
    header = open(os.path.join(ROOT, "include", "abs.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    names = set(re.findall(r"\b(abs_[a-z_]+)\s*\(", header))
    assert {"abs_create", "abs_round", "abs_get_model", "abs_trace", "abs_destroy"} <= names
    dll = ctypes.CDLL(lib.library_path())
    for n in sorted(names):
        assert hasattr(dll, n), n
    assert lib.abs_config_bytes() == ctypes.sizeof(lib.AbsConfig) == 152


def _dry_vs_oracle(p, T):
    d = workloads.make_inputs(p)
    o = AbsOracle(p, d["X"], d["y"], d["w0"], keep_models=False).run(T)
    Ks = [r["K"] for r in o.trace]
    q = dict(p, k_mode=2)
    sim = lib.Simulation(q, None, device_mode=0, k_replay=Ks)
    sim.round(T)
    got = sim.trace()
    sim.close()
    want = np.stack([trace_words(r, p["N"]) for r in o.trace])
    keep = np.ones(got.shape[1], bool)
    keep[10] = False          # the loss word: there are no losses without a device
    keep[11] = False          # K^{t+1}: in replay mode the last record repeats K
    assert np.array_equal(got[:, keep], want[:, keep])
    assert np.array_equal(got[:-1, 11], want[:-1, 11])
    return o


@pytest.mark.parametrize("i,over,T", [
    (1, dict(), 200),
    (2, dict(M=3200, dims=[16, 10]), 300),
    (3, dict(M=3200, dims=[16, 8, 10], lr=2e-3), 120),                     # slow subset
    (4, dict(M=6400, dims=[16, 8, 8, 10], lr=2e-3), 80),                   # staleness-aware step
    (5, dict(M=12800, dims=[16, 8, 8, 100], n_classes=100, lr=2e-3), 60),  # Pareto times, N = 128
    (1, dict(tau_mode=1, tau_cap=1), 150),
    (1, dict(tau_mode=2, tau_cap=40, k_mode=1, K0=1), 150),
    (1, dict(k_mode=3), 150),
])
def test_scheduler_trace_equals_oracle(i, over, T):
    p = workloads.scaled_preset(i, **over)
    o = _dry_vs_oracle(p, T)
    if over.get("tau_mode", 0) != 2:
        assert sum(r["n_restart"] for r in o.trace) > 0


def test_scheduler_equals_the_hand_worked_run():
    """The C++ scheduler against tests/golden/abs_hand_worked_schedule.txt (pencil-and-paper run of
    Algorithm 1: ties, a gradient of staleness tau_max + 1, a restart by Eq. 6)."""
    setting, want = hand_worked_schedule()
    p = workloads.scaled_preset(1, M=400, B=8, dims=[12, 1], **setting)
    sim = lib.Simulation(p, None, device_mode=0)
    sim.round(len(want))
    got = sim.trace()
    sim.close()
    for row, w in zip(got, want):
        K = w["K"]
        assert [int(row[0]), int(row[1]), int(row[2])] == [w["t"], K, w["tau_max"]]
        assert (int(row[3]) & 0xFFFFFFFF) | (int(row[4]) << 32) == w["now"]
        assert int(row[5]) == len(w["restart_ids"]) and int(row[6]) == w["comm_uploads"] and int(row[8]) == w["comm_restarts"]
        assert list(row[12:12 + K]) == w["ids"] and list(row[12 + K:12 + 2 * K]) == w["vers"]
        assert list(row[12 + 2 * K:12 + 3 * K]) == w["taus"]
        assert list(row[12 + 3 * K:12 + 3 * K + len(w["restart_ids"])]) == w["restart_ids"]


def test_draws_equal_oracle():
    for i in (1, 3, 5):
        p = workloads.scaled_preset(i, M=12800)
        cfg = lib.make_config(p)
        for n in (0, 1, p["N"] - 1):
            for j in (0, 1, 7, 1000):
                assert lib.abs_draw_time_ticks(cfg, n, j) == crng.compute_time_ticks(p, n, j)
                assert list(lib.abs_draw_batch_rows(cfg, n, j)) == crng.batch_indices(p, n, j)


def test_argument_errors():
    p = workloads.preset(1)
    with pytest.raises(lib.AbsError) as e:
        lib.Simulation(p, None, device_mode=0)              # adaptive K has no losses to use
    assert e.value.code == -1
    for bad in (dict(N=0), dict(N=129), dict(K0=9), dict(dims=[100, 2]), dict(lr=-1.0), dict(tau_cap=-1),
                dict(M=4)):
        q = dict(p, k_mode=1, **bad)
        with pytest.raises(lib.AbsError):
            lib.Simulation(q, None, device_mode=0)
    # replay array exhausted -> ABS_E_REPLAY, earlier rounds stay readable
    q = dict(p, k_mode=2)
    sim = lib.Simulation(q, None, device_mode=0, k_replay=[2, 3, 3])
    with pytest.raises(lib.AbsError) as e:
        sim.round(5)
    assert e.value.code == -6 and lib.abs_rounds_done(sim.handle) == 3
    assert sim.trace().shape == (3, lib.trace_stride(8))
    with pytest.raises(lib.AbsError):
        lib.abs_trace(sim.handle, 0, 4, 8)
    sim.close()
    # a worker staler than the ring allows is refused (tau_mode 2 with a small tau_cap)
    q = dict(p, k_mode=1, K0=1, tau_mode=2, tau_cap=0)
    sim = lib.Simulation(q, None, device_mode=0)
    with pytest.raises(lib.AbsError) as e:
        sim.round(200)
    assert e.value.code == -4
    sim.close()


def test_batch_and_evaluate_argument_errors_without_a_gpu():
    """Schedule-only handles have no model: they can be neither evaluated nor batched."""
    p = dict(workloads.preset(1), k_mode=1)
    a = lib.Simulation(p, None, device_mode=0)
    b = lib.Simulation(dict(p, seed_sim=7), None, device_mode=0)
    with pytest.raises(lib.AbsError) as e:
        lib.abs_evaluate(a.handle, -1, None, None, 10)
    assert e.value.code == -1
    with pytest.raises(lib.AbsError) as e:
        lib.abs_batch_create([a.handle, b.handle])
    assert e.value.code == -1 and "schedule-only" in str(e.value)
    with pytest.raises(lib.AbsError):
        lib.abs_batch_create([])
    assert lib.abs_batch_workspace_size([a.handle, b.handle]) == 0     # no batch, no size
    a.close(); b.close()


def test_workspace_of_local_sgd_holds_no_weight_gradient_partials():
    """U > 1 takes the step in the weight gradient's epilogue: beside what U = 1 needs without its partials (16 per layer)
    the workspace holds the uploads' private models, their losses and the averaged change, and nothing else."""
    up = lambda v, m: (v + m - 1) // m * m
    for dims, N in (([3072, 2048, 2048, 100], 128), ([200, 96, 10], 8)):
        p = workloads.scaled_preset(3, M=12800, dims=dims, n_classes=dims[-1], N=N, K0=2, n_slow=0)
        one, local = (lib.abs_workspace_size(lib.make_config(dict(p, U=U))) for U in (1, 10))
        pad = [up(d, 128) for d in dims]
        pad[-1] = 64 if dims[-1] <= 64 else pad[-1]
        layers = range(len(dims) - 1)
        partials = sum(pad[l] * (pad[l + 1] + 32) * 4 * 16 for l in layers)
        slot = up(sum(dims[l] * dims[l + 1] + dims[l + 1] for l in layers), 64) * 4
        shadow = up(sum(pad[l + 1] * (pad[l] + 64) + (pad[l] * (pad[l + 1] + 64) if l else 0) for l in layers), 128) * 2
        private = N * (slot + shadow + 4) + slot
        assert abs((local - (one - partials)) - private) <= 256 * 8, (dims, N, local, one, partials, private)


def test_a_row_pitch_without_room_for_the_zeros_does_not_compile():
    """Gathered rows read the pad behind a weight row as their zeros: a build with a shorter pad is refused."""
    import subprocess
    from paper_2301_08895_amd import build
    src = os.path.join(ROOT, "paper_2301_08895_amd", "csrc", "kernels_mlp.hip")
    for pad, ok in ((0, False), (32, False), (64, True), (128, True)):
        r = subprocess.run([build.hipcc(), "-x", "hip", "-std=c++17", "-fsyntax-only", "--cuda-host-only",
                            f"-DABS_PITCH_PAD={pad}", src], capture_output=True, text=True)
        assert (r.returncode == 0) == ok, (pad, r.stderr[-2000:])
        assert ok or "gathered k-step" in r.stderr


def test_workspace_of_the_convolutional_model_by_the_row():
    """What one more row of a minibatch costs; the gradient of the first pooled map is in memory only where the backward
    half's stages do not fit the LDS at once."""
    for (C0, S, C1, C2, F1, F2, C, k), apart in (((3, 32, 6, 16, 120, 84, 10, 5), False), ((4, 62, 10, 8, 24, 12, 4, 3), True)):
        p = workloads.scaled_preset(6, M=200_000, N=100, dims=[C0 * S * S, C1, C2, F1, F2, C, C0, k], n_classes=C)
        a, b = (lib.abs_workspace_size(lib.make_config(dict(p, B=B))) for B in (100, 200))
        S1 = (S - k + 1) // 2
        n1, F0 = C1 * S1 * S1, C2 * ((S1 - k + 1) // 2) ** 2
        grow = (C0 * k * k + 1) * C1 + (C1 * k * k + 1) * C2
        words = 3 + n1 + F0 + 2 * (F1 + F2) + C + F0 + grow + 2 + (n1 if apart else 0)
        assert abs((b - a) / 10_000 - (4 * words + n1 + F0)) < 1, (S, (b - a) / 10_000, 4 * words + n1 + F0)


@pytest.mark.parametrize("i", [1, 2, 3, 6])
def test_initial_weights_of_another_size_are_refused(i):
    """abs_create copies the model's parameters from w0: an array of another length is refused before anything touches a device."""
    small = dict(M=400) if i != 3 else dict(M=400, dims=[16, 24, 24, 4], n_classes=4, N=4, B=8, n_slow=1)
    p = workloads.scaled_preset(i, **small)
    d = workloads.make_inputs(p)
    assert lib.binding._model_size(p) == d["w0"].size == workloads.param_count(p)
    cases = [(p, dict(d, w0=d["w0"][:-1])), (p, dict(d, w0=np.concatenate([d["w0"], d["w0"][:1]])))]
    if i == 3:                                           # inputs made before the blocks were asked for
        q = workloads.with_blocks(p, groups=8)
        assert lib.binding._model_size(q) == workloads.make_inputs(q)["w0"].size == d["w0"].size + 2 * (24 + 24)
        cases += [(q, d), (p, workloads.make_inputs(q))]
    for q, wrong in cases:
        with pytest.raises(lib.AbsError) as e:
            lib.Simulation(q, wrong)
        assert e.value.code == -1 and "parameters" in str(e.value)
