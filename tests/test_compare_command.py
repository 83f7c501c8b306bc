"""The read-out command's choice of methods (no GPU: the runs themselves are replaced)."""
import pytest

from paper_2301_08895_amd import compare


def run(monkeypatch, *args):
    """(name, local steps, groups or None) of the methods that a command line runs."""
    import workloads
    seen = []

    def record(p, name, rounds, every, eval_rows, over):
        q = workloads.method_preset(p, name, **over)
        seen.append((name, q.get("U", 1), q["blocks"]["groups"] if q.get("blocks") else None))
        return []

    monkeypatch.setattr(compare, "run_method", record)
    assert compare.main(list(args)) == 0
    return seen


def test_blocks_by_default_run_every_method_of_one_local_step(monkeypatch):
    got = run(monkeypatch, "--config", "3", "--blocks", "16", "--dropout", "0.2")
    assert got == [(n, 1, 16) for n in ("abs", "adasync", "sa_adasync", "k_async")]
    assert run(monkeypatch, "--config", "3", "--blocks", "16", "--methods", "sync_sgd,asgd") == [("sync_sgd", 1, 16), ("asgd", 1, 16)]
    assert run(monkeypatch, "--config", "3", "--blocks", "16", "--U", "1")[-1] == ("local_sgd", 1, 16)


@pytest.mark.parametrize("args", [("--methods", "abs,local_sgd"), ("--U", "2"), ("--methods", "k_async", "--U", "3")])
def test_blocks_of_several_local_steps_are_refused_before_a_round(monkeypatch, capsys, args):
    with pytest.raises(SystemExit):
        run(monkeypatch, "--config", "3", "--blocks", "16", *args)
    assert "one local step" in capsys.readouterr().err


def test_other_networks_keep_their_methods(monkeypatch):
    assert [n for n, _, _ in run(monkeypatch, "--config", "2")] == ["abs", "adasync", "sa_adasync", "k_async", "local_sgd"]
    assert run(monkeypatch, "--config", "2", "--U", "4", "--methods", "abs,sync_sgd") == [("abs", 4, None), ("sync_sgd", 1, None)]
