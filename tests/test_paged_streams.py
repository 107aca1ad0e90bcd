"""PagedStreams' book of pages on the host: a step that does not return a batch changes nothing."""
import pytest

from paper_2605_09681_amd.layer import PagedStreams


def book(p):
    return list(p._free), {s: list(v) for s, v in p._pages.items()}, dict(p._len)


@pytest.mark.parametrize("new,error", [
    ([(1, 20), (2, 1)], ValueError),                # (host tensors: the batch is refused)
    ([(1, 20), (2, 1.5)], TypeError), ([(1, 20), (2, "3")], TypeError), ([(1, 20), (9, 1)], KeyError),
    ([(1, 20), (2, 80)], RuntimeError), ([(1, 20), (2, -1)], ValueError)])
def test_a_step_that_fails(new, error):
    p = PagedStreams(1, 2, 64, n_pages=6, page_tokens=16, device="cpu")
    assert [p.open(), p.open()] == [1, 2]
    before = book(p)
    with pytest.raises(error):
        p.step(new)
    assert book(p) == before


def test_a_batch_that_cannot_be_made(monkeypatch):
    from paper_2605_09681_amd import layer
    p = PagedStreams(1, 2, 64, n_pages=6, page_tokens=16, device="cpu")
    s = p.open()

    def make(table, lens, starts, page_tokens, n_tokens, max_new, sum_len):
        return table.tolist(), lens.tolist(), starts.tolist(), page_tokens, n_tokens, max_new, sum_len
    monkeypatch.setattr(layer, "PagedBatch", make)
    assert p.step([(s, 20)]) == ([[0, 1]], [20], [0, 20], 16, 20, 20, 20)
    t = p.open()
    assert p.step([(t, 17), (s, 12)]) == ([[2, 3], [0, 1]], [17, 32], [0, 17, 29], 16, 29, 17, 49)
    before = book(p)

    def refuse(*args):
        raise RuntimeError("no memory for the tables")
    monkeypatch.setattr(layer, "PagedBatch", refuse)
    with pytest.raises(RuntimeError):
        p.step([(t, 30), (s, 1)])
    assert book(p) == before
    monkeypatch.setattr(layer, "PagedBatch", make)
    assert p.step([(s, 1), (t, 15)]) == ([[0, 1, 4], [2, 3, -1]], [33, 32], [0, 1, 16], 16, 16, 15, 65)
    p.close(s)
    assert len(p._free) == 4
