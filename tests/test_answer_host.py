"""Host-side parts of the answers (no GPU): drafts from the text itself, and refusals before any buffer is made."""
import pytest

from paper_2609_34977_gb300.answer import TreeAnswer, ngram_drafts


def test_ngram_drafts_continue_the_last_occurrence():
    text = [7, 1, 2, 9, 1, 2, 3, 4, 5, 1, 2]
    assert ngram_drafts(text, 4) == [(3, 0), (4, 1), (5, 2), (1, 3)]
    assert ngram_drafts(text, 1) == [(3, 0)]
    assert ngram_drafts([1, 2, 3], 4) == []            # the last two tokens occur once
    assert ngram_drafts([5], 4) == [] and ngram_drafts([], 4) == []
    assert ngram_drafts([4, 4, 4], 3) == [(4, 0)]      # the occurrence may overlap the end


@pytest.mark.parametrize("kw", [dict(budget=30, n_sink=4, n_recent=32), dict(budget=120, max_nodes=16), dict(budget=0)])
def test_a_budget_needs_room(kw):
    class Model:
        cfg = dict(n_layers=1, n_kv_heads=1, head_dim=64, n_heads=1, vocab=8, d_model=64)
    with pytest.raises(ValueError, match="budget"):
        TreeAnswer(Model, None, 1, 128, **kw)


def test_ngram_drafts_stop_at_an_images_placeholders():
    text = [1, 2, 3, -1, -1, 4, 1, 2]
    assert ngram_drafts(text, 5) == [(3, 0), (-1, 1), (-1, 2), (4, 3), (1, 4)]
    assert ngram_drafts(text, 5, vocab=8) == [(3, 0)] and ngram_drafts(text, 5, vocab=3) == []


def test_the_embedding_is_the_vocabulary_s():
    class Model:
        cfg = dict(n_layers=1, n_kv_heads=1, head_dim=64, n_heads=1, vocab=8, d_model=64)

    class Embed:
        shape = (7, 64)
    with pytest.raises(ValueError, match="embed"):
        TreeAnswer(Model, Embed, 1, 128)
