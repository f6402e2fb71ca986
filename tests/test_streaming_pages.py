"""Which pages StreamingGlobalAttention gives its sequence, and what a step that fails leaves behind, on stand-ins for the context and the
cache.  No GPU."""
import types

import pytest
import torch

from paper_2512_04939_b200 import streaming

DIM, HEADS = 1024, 16


class Cache:
    """Notes which tokens lie in which pages, as the pool would hold them."""

    fail = None  # the call that raises

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype, device):
        c = cls()
        c.pages, c.page_size, c.pool = pages, page_size, {}
        return c

    def _called(self, name):
        if Cache.fail == name:
            raise RuntimeError(name)

    def batch(self, rows, lengths, pages, causal_block=0):
        self._called("batch")
        assert len(pages[0]) == -(-lengths[0] // self.page_size) and len(set(pages[0])) == len(pages[0])
        assert all(0 <= p < self.pages for p in pages[0])
        return types.SimpleNamespace(rows=rows[0], length=lengths[0], pages=list(pages[0]))

    def append(self, batch, k, v):
        self._called("append")
        for i in range(batch.rows):
            at = batch.length - batch.rows + i
            self.pool[batch.pages[at // self.page_size], at % self.page_size] = int(k[i, 0, 0])

    def attend(self, batch, q):
        self._called("attend")
        self.seen = [self.pool[batch.pages[i // self.page_size], i % self.page_size] for i in range(batch.length)]
        return q


class Context:
    cfg, dim, device = types.SimpleNamespace(heads=HEADS), DIM, torch.device("cpu")

    def linear(self, a, w, bias=None):
        if Cache.fail == ("linear", w.shape[0]):
            raise RuntimeError("linear")
        return a.repeat(1, 3) if w.shape[0] == 3 * DIM else a


@pytest.fixture
def made(monkeypatch):
    monkeypatch.setattr(streaming, "KVCache", Cache)
    monkeypatch.setattr(Cache, "fail", None)
    return lambda *a, **k: streaming.StreamingGlobalAttention(Context(), *a, **k)


WEIGHTS = [torch.zeros(3 * DIM, DIM, dtype=torch.bfloat16), None, torch.zeros(DIM, DIM, dtype=torch.bfloat16), None]


def tokens(first, n):
    """Rows that say which token they are (numbers that bfloat16 holds)."""
    return torch.arange(first, first + n).remainder(256)[:, None].expand(n, DIM).bfloat16().contiguous()


def whole(layer):
    """Every page is with the sequence or free."""
    return sorted(layer.pages + layer.free) == list(range(layer.cache.pages)) and len(layer.pages) == -(-layer.length // layer.cache.page_size)


@pytest.mark.parametrize("page_size", [16, 64])
@pytest.mark.parametrize("window,capacity", [(128, 128), (100, 100), (1, 1), (1, 70), (65, 100), (130, 200)])
@pytest.mark.parametrize("chunks", [[1] * 400, [100] * 9, [37, 1, 63, 64, 65, 5, 70] * 4])
def test_a_window_that_fits_never_runs_out_of_pages(made, window, capacity, page_size, chunks):
    layer, at = made(capacity, page_size=page_size, window=window), 0
    for n in chunks:
        n = min(n, capacity)
        layer.step(tokens(at, n), *WEIGHTS)
        at += n
        held = min(at, max(window, n))
        assert held <= layer.length < held + page_size and whole(layer)
        assert layer.cache.seen == [i % 256 for i in range(at - layer.length, at)]


@pytest.mark.parametrize("window", [None, 100])
@pytest.mark.parametrize("fail", [("linear", 3 * DIM), "batch", "append", "pages"])
def test_a_step_that_fails_before_its_rows_are_stored_changes_nothing(made, window, fail):
    """Whatever raises - a projection, the plan, the store, or the lack of pages - the next step goes on from where the last one ended."""
    layer = made(200, page_size=16, window=window)
    for at in range(0, 180, 30):
        layer.step(tokens(at, 30), *WEIGHTS)
    before = list(layer.pages), list(layer.free), layer.length
    with pytest.raises(ValueError if fail == "pages" else RuntimeError):
        if fail == "pages":
            layer.step(tokens(180, 300), *WEIGHTS)
        else:
            Cache.fail = fail
            layer.step(tokens(180, 17), *WEIGHTS)
    Cache.fail = None
    assert (layer.pages, layer.free, layer.length) == before
    layer.step(tokens(180, 17), *WEIGHTS)
    assert layer.cache.seen == [i % 256 for i in range(197 - layer.length, 197)] and whole(layer)


@pytest.mark.parametrize("fail", ["attend", ("linear", DIM)])
def test_rows_that_are_stored_stay(made, fail):
    """What raises behind the store leaves the new rows in the sequence."""
    layer = made(200, page_size=16, window=100)
    layer.step(tokens(0, 90), *WEIGHTS)
    Cache.fail = fail
    with pytest.raises(RuntimeError):
        layer.step(tokens(90, 40), *WEIGHTS)
    Cache.fail = None
    assert whole(layer)
    layer.step(tokens(130, 1), *WEIGHTS)
    assert layer.cache.seen == [i % 256 for i in range(131 - layer.length, 131)] and layer.length >= 100


def bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


@pytest.mark.parametrize("which,bad", [
    (0, bf(3, DIM - 64)), (0, bf(3, 2 * DIM)[:, ::2]), (0, torch.zeros(3, DIM)), (0, bf(3, 1, DIM)), (0, bf(0, DIM)), (0, bf(3, DIM).to("meta")),
    (1, bf(3 * DIM, DIM - 64)), (1, bf(2 * DIM, DIM)), (1, bf(4 * DIM, DIM)), (1, torch.zeros(3 * DIM, DIM)), (1, bf(DIM, 3 * DIM).t()), (1, None),
    (2, bf(DIM)), (2, bf(3 * DIM, 1)), (2, torch.zeros(3 * DIM)), (3, bf(DIM, DIM - 1)), (3, bf(2 * DIM, DIM)), (3, bf(DIM, DIM).to("meta")), (3, None), (4, bf(DIM - 1))])
def test_operands_that_the_projections_cannot_take_are_refused(made, which, bad):
    """The matrix product is told sizes and trusts every extent: what is smaller than them would be read past its end."""
    layer = made(100)
    args = [tokens(0, 3), *WEIGHTS]
    args[which] = bad
    with pytest.raises(ValueError):
        layer.step(*args)
    assert layer.length == 0
    layer.step(tokens(0, 3), WEIGHTS[0], bf(3 * DIM), WEIGHTS[2], bf(DIM))
