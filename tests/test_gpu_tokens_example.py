"""The token mixer of examples/token_mixer.py: it learns, and sampling continues what the prompt left."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_mixer.py")
    spec = importlib.util.spec_from_file_location("token_mixer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_learns(ex):
    """A guess at 12 symbols costs log 12 = 2.48; the sequences' first periods cannot be known, the rest can."""
    _, losses, _ = ex.train(steps=60, log=lambda *a, **k: None)
    assert 2.2 < losses[0] < 3.2 and sum(losses[-5:]) / 5 < 1.6, losses


def test_tokens_one_by_one_are_the_whole_sequence(ex):
    """The logits behind token t, from a prompt of lens[b] tokens and single tokens after it, are those of the whole sequence;
    bfloat16 throughout, so to a few of its roundings (2^-8) of logits of size one."""
    torch.manual_seed(1)
    model = ex.Mixer(12).to(ex.DEV)
    seq = ex.batch(4, 30, 12, torch.Generator().manual_seed(2))
    with torch.no_grad():
        whole = model(seq).float()
    lens = torch.tensor([20, 1, 17, 16], dtype=torch.int32, device=ex.DEV)
    at = lens.long().clone()
    logits, state = model.prompt(seq[:, :20].contiguous(), lens)
    rows = torch.arange(4, device=ex.DEV)
    for _ in range(8):
        assert (logits.float() - whole[rows, at - 1]).abs().max() < 0.06
        logits = model.next(seq[rows, at], state)
        at += 1
