"""Options of the word_model command that are refused before anything is fitted, without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2007_08725_amd import word_model  # noqa: E402

BAD = [["--distil", "0.5"], ["--reader", "--distil", "-0.1"], ["--reader", "--distil", "1.01"],
       ["--reader", "--distil", "nan"], ["--top", "8"], ["--reader", "--top", "8"], ["--temperature", "2"],
       ["--reader", "--temperature", "2"], ["--reader", "--distil", "0", "--top", "8"],
       ["--reader", "--distil", "0.5", "--top", "0"], ["--reader", "--distil", "0.5", "--top", "257"],
       ["--reader", "--distil", "0.5", "--temperature", "0"], ["--reader", "--distil", "0.5", "--temperature", "-1"],
       ["--reader", "--distil", "0.5", "--temperature", "nan"], ["--reader", "--distil", "0.5", "--temperature", "inf"],
       ["--reader", "--distil", "0.5", "--temperature", "1e-320"],
       ["--reader", "--distil", "0.5", "--temperature", "1e-39"], ["--reader", "--distil", "0.5", "--temperature", "1e39"]]


@pytest.mark.parametrize("args", BAD, ids=" ".join)
def test_refused(args, capsys):
    with pytest.raises(SystemExit) as e:
        word_model.main(args)
    assert e.value.code == 2 and "--" in capsys.readouterr().err.splitlines()[-1]


class Reached(Exception):
    pass


@pytest.mark.parametrize("args", [[], ["--reader"], ["--reader", "--distil", "0"], ["--reader", "--distil", "1"],
                                  ["--reader", "--distil", "0.5", "--top", "256", "--temperature", "0.5"]])
def test_accepted(args, monkeypatch):
    """The first thing that the command does after its checks is to take the device."""
    def reached(device):
        raise Reached

    monkeypatch.setattr(torch.cuda, "set_device", reached)
    with pytest.raises(Reached):
        word_model.main(args)
