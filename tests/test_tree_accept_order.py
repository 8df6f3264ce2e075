"""PagedCache.accept beside calls that are refused: what is open, and what is left as it was.  Without a GPU."""
import pytest
import torch

from paper_2603_06274_amd import decode_binding as db
from paper_2603_06274_amd import tree_binding as tb
from paper_2603_06274_amd.decode import PagedCache

from test_norm_tree_host import here, whole       # noqa: F401

TABLE = db.stem_block_table


@pytest.fixture
def calls(here, monkeypatch):                     # noqa: F811
    """What reaches the library."""
    made = []
    monkeypatch.setattr(db, "stem_block_table", lambda *a: made.append("table"))
    monkeypatch.setattr(tb, "stem_tree_accept", lambda *a: made.append("accept"))
    monkeypatch.setattr(tb, "stem_tree_commit", lambda *a: made.append("commit"))
    return made


def test_a_step_that_is_refused_opens_nothing(calls, monkeypatch):
    cache, x = PagedCache(2, 4, 16, 2, 1, 64, tokens=4, device="cpu"), whole(4)
    cache.advance(None, 2)
    cache.accept(x, x, x)
    monkeypatch.setattr(db, "stem_block_table", TABLE)
    with pytest.raises(ValueError, match="new_lens"):
        cache.advance(x.double(), 3)
    assert cache.shape.c.max_new == 2
    with pytest.raises(RuntimeError, match="no step"):
        cache.accept(x, x, x)
    assert calls == ["table", "accept", "commit"]


@pytest.mark.parametrize("d,heads,dtype", [(100, 1, torch.bfloat16), (1032, 1, torch.bfloat16), (64, 1, torch.float64),
                                           (1024, 32769, torch.bfloat16), (1024, 16385, torch.float32)])
def test_pages_whose_rows_cannot_be_moved(calls, d, heads, dtype):
    """Refused before the books change."""
    cache, x = PagedCache(2, 4, 16, 2, 1, d, tokens=4, dtype=dtype, device="cpu"), whole(4)
    cache.pages.heads = heads                     # (rows of 64 MiB and more, without their memory)
    cache.advance(None, 2)
    with pytest.raises(ValueError, match="moved"):
        cache.accept(x, x, x)
    assert calls == ["table"]


def test_a_refused_acceptance_can_be_tried_again(calls):
    """Once accept_refused has said that it was refused, and only then."""
    cache, x = PagedCache(2, 4, 16, 2, 1, 64, tokens=4, device="cpu"), whole(4)
    assert cache.accept_refused() == (0, 0)
    with pytest.raises(RuntimeError):
        cache.accept(x, x, x)                     # (there is no step)
    for why in ((1, 0), (0, 2)):
        cache.advance(None, 2)
        cache.accept(x, x, x)
        cache.accept_status.copy_(torch.tensor(why))
        with pytest.raises(RuntimeError):
            cache.accept(x, x, x)                 # (nobody has asked)
        assert cache.accept_refused() == why
        cache.accept(x, x, x)
        cache.accept_status.zero_()
        assert cache.accept_refused() == (0, 0)
        with pytest.raises(RuntimeError):
            cache.accept(x, x, x)


def test_replayed_steps_may_have_more_new_tokens_than_the_last_call(calls, monkeypatch):
    """Where steps or acceptances are in graphs, an acceptance is of whichever step has been replayed: of as many tokens as there are rows."""
    asked = []
    monkeypatch.setattr(tb, "stem_tree_accept", lambda shape, *a: asked.append(shape.c[torch.int32].max_new))
    x = whole(4)
    for captured in ("step", "accept", None):
        cache = PagedCache(2, 4, 16, 2, 1, 64, tokens=4, device="cpu")
        cache._capturing = lambda: captured == "step"
        cache.advance(None, 3)
        cache._capturing = lambda: False
        cache.advance(None, 1)
        cache._capturing = lambda: captured == "accept"
        cache.accept(x, x, x)
    cache.advance()                                # any number of new tokens
    cache.accept(x, x, x)
    large = PagedCache(2, 200, 16, 100, 1, 64, tokens=2000, device="cpu")
    large.advance()
    large.accept(*[whole(2000)] * 3)
    assert asked == [4, 4, 1, 4, tb.STEM_MAX_TREE]
