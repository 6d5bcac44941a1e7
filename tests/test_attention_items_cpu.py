"""How the warps of the attention's persistent kernels pass items on, as a model on the host: items come through four places, each
free again once every reader has passed it, and empty items (nothing but padding) lie between others in any number. The model
has the waits of the forward pass (csrc/k_attention_tc.cu) and of the dQ kernel (csrc/k_attention_grad_tc.cu); how far the MMAs'
warp looks ahead while products of a tile are still to be issued is read from their source."""
import random

import pytest

from test_kernel_source_cpu import block, source

PLACES = 4


def looks_ahead(name, walk):
    """1: at the item right behind only; None: past any number of empty items."""
    text = source(name)
    body, _ = block(text, text.index(f"struct {walk} {{"))
    held = "if (busy) break;" in body and "then.next(now.valid, bars," in text
    return 1 if held else None


class Model:
    """Roles are generators that yield a condition to wait for; run() steps them until all are done or none can go on."""

    def __init__(self, items, ahead, forward):
        self.items, self.ahead, self.forward = items, ahead, forward  # items: per item the numbers of key tiles of its two parts
        self.made, self.passed = 0, {}
        self.queries = [-1, -1]     # the item whose queries a part has, and whose scores have been issued in full
        self.scored = [set(), set()]
        self.weighed, self.summed, self.out = [set(), set()], [set(), set()], [set(), set()]

    def any(self, r):
        return any(self.items[r])

    def read(self, who, r):
        yield lambda: self.made > r
        self.passed[who] = r + 1

    def maker(self):
        last = [None, None]
        for r in range(len(self.items) + 1):
            if r < len(self.items):
                yield lambda r=r: r < PLACES or min(self.passed.values()) > r - PLACES
                self.made = r + 1
            if r:
                for w, tiles in enumerate(self.items[r - 1]):
                    if tiles:
                        before = last[w]
                        yield lambda w=w, before=before: before is None or before in self.scored[w]
                        self.queries[w] = last[w] = r - 1

    def loads(self):
        for r in range(len(self.items)):
            yield from self.read("loads", r)

    def rows(self, w):
        yield from self.read(f"rows{w}", 0)
        before = None
        for r in range(len(self.items)):
            if self.forward and r + 1 < len(self.items):
                yield from self.read(f"rows{w}", r + 1)
            if self.items[r][w]:
                yield lambda r=r: r in self.scored[w]  # of its last tile; those before come with it
                if self.forward:
                    yield lambda before=before: before is None or before in self.out[w]
                self.summed[w].add(r)
                before = r
            if not self.forward:
                if r + 1 < len(self.items):
                    yield from self.read(f"rows{w}", r + 1)
                if self.items[r][w]:
                    yield lambda r=r: r in self.weighed[w]
                    self.out[w].add(r)

    def outputs(self):
        for r in range(len(self.items)):
            yield from self.read("outputs", r)
            for w, tiles in enumerate(self.items[r]):
                if tiles:
                    yield lambda r=r, w=w: r in self.summed[w] and r in self.weighed[w]
                    self.out[w].add(r)

    def mmas(self):
        r, now = 0, None
        while True:
            then = None
            while r < len(self.items) and then is None:
                yield from self.read("mmas", r)
                then, r = (r if self.any(r) else None), r + 1
                if now is not None and self.ahead == 1:
                    break
            if now is None and then is None:
                return
            for w in (0, 1):
                if self.forward:  # P V of `now`, then S of `then`, for either part
                    if now is not None and self.items[now][w]:
                        self.weighed[w].add(now)
                    if then is not None and self.items[then][w]:
                        yield lambda w=w, then=then: self.queries[w] >= then
                        self.scored[w].add(then)
                else:  # S of `then`, then dQ of `now`
                    if then is not None and self.items[then][w]:
                        yield lambda w=w, then=then: self.queries[w] >= then
                        self.scored[w].add(then)
                    if now is not None and self.items[now][w]:
                        yield lambda w=w, now=now: now in self.summed[w]
                        self.weighed[w].add(now)
            now = then

    def run(self):
        roles = [self.maker(), self.loads(), self.rows(0), self.outputs(), self.mmas()] + ([self.rows(1)] if self.forward else [])
        readers = ["loads", "rows0", "outputs", "mmas"] + (["rows1"] if self.forward else [])
        self.passed = {x: 0 for x in readers}
        waits = {}
        for g in roles:
            waits[g] = next(g, None)
        while True:
            moved = False
            for g in roles:
                while waits[g] is not None and waits[g]():
                    waits[g], moved = next(g, None), True
            if all(x is None for x in waits.values()):
                return True
            if not moved:
                return False


def sequences():
    rng = random.Random(3)
    for empty in range(0, 12):
        yield [True] + [False] * empty + [True] * 3
    for share in (0.1, 0.5, 0.9):
        for _ in range(40):
            yield [rng.random() >= share for _ in range(30)]


@pytest.mark.parametrize("name,walk,forward", [("k_attention_tc.cu", "Walk", True), ("k_attention_grad_tc.cu", "DqWalk", False)])
def test_empty_items_lock_nobody_out(name, walk, forward):
    ahead = looks_ahead(name, walk)
    for i, any_keys in enumerate(sequences()):
        items = []
        for k, live in enumerate(any_keys):  # of one part, the other, or both
            one = (k + i) % 3
            items.append((int(live and one != 0), int(live and one != 1)) if forward else (int(live), 0))
        assert Model(items, ahead, forward).run(), f"locked up: {items}"


def test_the_model_sees_the_lock():
    """Looking past empty items without end locks up at three of them."""
    for forward in (True, False):
        part = (1, 1) if forward else (1, 0)
        assert Model([part] + [(0, 0)] * 2 + [part], None, forward).run()
        assert not Model([part] + [(0, 0)] * 4 + [part], None, forward).run()
