"""The controller's option for evaluation in 4 bits, without a GPU."""
import pytest


@pytest.fixture(scope="module")
def C():
    from paper_2102_08550_amd import controller
    return controller


def test_command_line_takes_the_4_bit_evaluation(C, monkeypatch, capsys):
    seen = []
    monkeypatch.setattr(C, "compare", lambda cfg, schedule, budget, **kw: seen.append(kw) or {})
    assert C.main(["--budget", "10"]) == 0
    assert C.main(["--mx4-eval", "--int8-eval"]) == 0
    capsys.readouterr()
    assert seen[0]["mx4_eval"] is False
    assert seen[1]["mx4_eval"] is True and seen[1]["int8_eval"] is True
    monkeypatch.setattr(C, "run_measured", lambda *a, **kw: pytest.fail("run"))
    with pytest.raises(SystemExit):
        C.main(["--measured", "2", "--mx4-eval"])
    assert "--mx4-eval" in capsys.readouterr().err


def test_a_convolutional_model_is_refused(C, monkeypatch):
    """By name and before anything is made or run."""
    import workload
    cfg = workload.Config("small-cnn", (8 * 8 * 3, 10), workload.FP32, K=1, n_rows=10, batch=4,
                          tau_rule="given", tau_given=(1,), image=(8, 8, 3), conv=((16, 1),))
    sched = C.SpeedSchedule([1])
    monkeypatch.setattr(workload, "gen_dataset", lambda cfg: pytest.fail("data made"))
    with pytest.raises(ValueError, match="fully connected"):
        C.run_paradigm(cfg, None, None, None, "bsp", sched, 1.0, 1.0, mx4_eval=True)
    with pytest.raises(ValueError, match="fully connected"):
        C.compare(cfg, sched, 1.0, mx4_eval=True)


def test_model_calls_refuse_null():
    import ctypes

    import paper_2102_08550_amd as P
    lib = P._lib()
    loss, hits = ctypes.c_double(), ctypes.c_int64()
    assert lib.oscars_micro_model_bytes(None) == 0
    assert lib.oscars_quantize_model_micro(None, 16, 16) == P.E_INVALID
    assert lib.oscars_evaluate_micro(None, 16, 16, 16, 1, ctypes.byref(loss),
                                     ctypes.byref(hits)) == P.E_INVALID
