"""The word reader's gradients of both of its losses (paper_2007_08725_amd/word_reader.py)."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_word_reader import batch_of, corpus  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_weight_gradients_are_added_in_single_precision(corpus, dtype):  # noqa: F811
    """The sum of the two losses' gradients is not rounded to the products' type once more."""
    from paper_2007_08725_amd import ops
    from paper_2007_08725_amd.word_reader import WordReader
    words, offsets, teacher = batch_of(corpus, 3, 8)
    rows = words.shape[0]
    model = WordReader(corpus[0].V, 40, 48, dtype=dtype)
    dloss, dapart = torch.linspace(-1, 1, rows, device="cuda"), torch.linspace(1, 0.2, rows, device="cuda")
    _, _, forward = model.loss(words, offsets, teacher, 1.5)
    got = model.gradients(forward, dloss, dapart)["weight"]
    p, h, lse, taught = forward[0], forward[-3], forward[-2], forward[-1]
    one = ops.softmax_xent_backward(dloss, lse, h, p["weight"], words, p["bias"])[1]
    two = ops.softmax_distill_backward(dapart, *taught)[1]
    assert got.dtype == torch.float32 and torch.equal(got, one.float() + two.float())


def test_the_command_says_what_the_reader_is_scored_on(capsys):
    import json
    from paper_2007_08725_amd import word_model
    assert word_model.main(["--docs", "60", "--iters", "2", "--steps", "2", "--batch", "256", "--hidden", "16",
                            "--reader", "--distil", "0.3", "--top", "4", "--temperature", "2"]) == 0
    said = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert said["llpt_reader"] < 0 and "trained on" in said["llpt_reader_of"]
