"""The drafting example refuses sizes that it cannot run, before it asks for a
GPU."""
import pytest

from examples import draft_and_verify as ex


@pytest.mark.parametrize("args", [
    ["--draft", "0"], ["--draft", "65"], ["--new", "0"], ["--seqs", "0"],
    ["--budget", "0", "--window", "0"], ["--budget", "-1"],
    ["--temperature", "0"]])
def test_command(args, capsys):
    with pytest.raises(SystemExit):
        ex.main(args)
    assert args[0][2:] in capsys.readouterr().err


def test_generate():
    for kw in (dict(new=0), dict(new=4, draft=0), dict(new=4, draft=65),
               dict(new=4, budget=0, window=0), dict(new=4, temperature=0.0)):
        with pytest.raises(ValueError):
            ex.generate(None, [[1, 2]], **kw)
    for prompts in ([], [[1], []]):
        with pytest.raises(ValueError):
            ex.generate(None, prompts, 4)
