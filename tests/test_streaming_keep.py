"""What StreamingGlobalAttention keeps when it is full, on stand-ins for the context and the cache.  No GPU."""
import pytest
import torch

import test_streaming_pages as base
from paper_2512_04939_b200 import streaming
from test_streaming_pages import WEIGHTS, Context, tokens, whole


class Cache(base.Cache):
    """Tokens draw as much as their own number modulo 7 says; all heads are alike."""

    @classmethod
    def empty(cls, pages, page_size, kv_heads, head_dim, dtype, device, weights=False):
        assert weights
        return super().empty(pages, page_size, kv_heads, head_dim, dtype, device)

    def evict(self, batch, into, first, last):
        self._called("evict")
        assert batch.rows == 0 and into.rows == into.length and not set(batch.pages) & set(into.pages)
        held = [self.pool[batch.pages[i // self.page_size], i % self.page_size] for i in range(batch.length)]
        middle = sorted(range(first, len(held) - last), key=lambda i: (-(held[i] % 7), i))[:into.length - first - last]
        kept = [*range(first), *sorted(middle), *range(len(held) - last, len(held))]
        for slot, i in enumerate(kept):
            self.pool[into.pages[slot // self.page_size], slot % self.page_size] = held[i]
        return torch.tensor(kept)[:, None]

    def attend(self, batch, q, lse):
        assert lse
        return super().attend(batch, q), "lse"

    def weigh(self, batch, q, lse, decay):
        self._called("weigh")
        assert lse == "lse" and decay == 0.5


@pytest.fixture
def made(monkeypatch):
    monkeypatch.setattr(streaming, "KVCache", Cache)
    monkeypatch.setattr(base.Cache, "fail", None)
    return lambda *a, **k: streaming.StreamingGlobalAttention(Context(), *a, **k)


def kept_of(held, keep, first, recent):
    middle = sorted(range(first, len(held) - recent), key=lambda i: (-(held[i] % 7), i))[:keep - first - recent]
    return held[:first] + [held[i] for i in sorted(middle)] + held[len(held) - recent:]


@pytest.mark.parametrize("page_size", [16, 64])
@pytest.mark.parametrize("capacity,keep,first,recent", [(200, 100, 5, 40), (130, 1, 0, 0), (101, 100, 0, 100), (300, 64, 64, 0)])
@pytest.mark.parametrize("chunks", [[1] * 700, [37, 1, 63, 64, 29] * 9])
def test_what_stays(made, capacity, keep, first, recent, chunks, page_size):
    layer, at, held = made(capacity, page_size=page_size, keep=keep, first=first, recent=recent, decay=0.5), 0, []
    for n in chunks:
        n = min(n, capacity - keep)
        if len(held) + n > capacity:
            held = kept_of(held, keep, first, recent)
        held = held + [i % 256 for i in range(at, at + n)]
        layer.step(tokens(at, n), *WEIGHTS)
        at += n
        assert layer.cache.seen == held and layer.length == len(held) and whole(layer)
    assert layer.kept is None if at <= capacity else layer.kept.shape == (keep, 1)
    layer.reset()
    assert layer.kept is None and layer.length == 0 and whole(layer)


@pytest.mark.parametrize("fail", [("linear", 3 * base.DIM), "batch", "evict", "append", "rows"])
def test_a_step_that_fails_before_its_rows_are_stored_changes_nothing(made, fail):
    layer = made(200, page_size=16, keep=100, first=3, recent=20, decay=0.5)
    for at in range(0, 190, 19):
        layer.step(tokens(at, 19), *WEIGHTS)
    before = list(layer.pages), list(layer.free), layer.length
    with pytest.raises(ValueError if fail == "rows" else RuntimeError):
        if fail == "rows":
            layer.step(tokens(190, 101), *WEIGHTS)
        else:
            base.Cache.fail = fail
            layer.step(tokens(190, 30), *WEIGHTS)
    base.Cache.fail = None
    assert (layer.pages, layer.free, layer.length) == before and layer.kept is None
    layer.step(tokens(190, 30), *WEIGHTS)
    assert layer.cache.seen == kept_of(list(range(190)), 100, 3, 20) + list(range(190, 220)) and whole(layer)


@pytest.mark.parametrize("kw", [dict(keep=200), dict(keep=0), dict(keep=100, window=50), dict(keep=100, first=60, recent=41), dict(keep=100, first=-1),
                                dict(keep=100, decay=1.5), dict(first=3), dict(recent=3), dict(decay=0.5)])
def test_refusals(made, kw):
    with pytest.raises(ValueError):
        made(200, **kw)


def test_positions_go_with_a_rotary(made):
    layer = made(200, keep=100, decay=0.5)
    with pytest.raises(ValueError):
        layer.step(tokens(0, 3), *WEIGHTS, positions=torch.zeros(3, 3, dtype=torch.int32))
    assert layer.length == 0
