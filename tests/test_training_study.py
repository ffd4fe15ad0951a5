"""The study's arguments, refused before anything touches a GPU."""
import pytest

pytest.importorskip("torch")


@pytest.mark.parametrize("bad", [dict(workers=0), dict(workers=17), dict(supersteps=0), dict(lookahead=0), dict(lookahead=-3)])
def test_a_run_of_nothing_is_refused(bad):
    from paper_2001_01347_amd import training_study
    with pytest.raises(ValueError):
        training_study.train(**{**dict(workers=4, supersteps=2, lookahead=3), **bad})


@pytest.mark.parametrize("args", [["--supersteps", "0"], ["--lookahead", "0"], ["--workers", "17"]])
def test_the_command_says_so(args, monkeypatch, capsys):
    from paper_2001_01347_amd import training_study
    monkeypatch.setattr("sys.argv", ["training_study", *args])
    with pytest.raises(SystemExit) as end:
        training_study.main()
    assert end.value.code == 2 and args[0] in capsys.readouterr().err
