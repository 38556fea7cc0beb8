"""The packed path's operand ring, modelled: the producer fills the stages of 8-bit blocks, the expanders those of 4-bit blocks from a ring of two raw
tiles, the MMA warp consumes them in order.  A wait knows only a parity, so it is right only where its barrier is in the phase
before the one that is waited for."""
import random

import pytest

RAW = 2


class Barrier:
    def __init__(self):
        self.done = 0                      # completed phases

    def passes(self, phase):               # mbarrier try_wait.parity: the phase of this parity is the last completed one
        return (self.done & 1) != (phase & 1)


def run(low, high, tiles, stages, rng):
    """True if no wait passed before its phase was complete."""
    blocks = ([0] * low + [1] * high) * tiles
    full, empty, raw_full, raw_empty = ([Barrier() for _ in range(n)] for n in (stages, stages, RAW, RAW))
    pending, sound = [], True

    def wait(bar, phase):                  # phase -1: nothing to wait for
        nonlocal sound
        while not bar.passes(phase):
            yield
        sound &= bar.done > phase

    def producer():
        lows = 0
        for i, high_block in enumerate(blocks):
            s, n = i % stages, i // stages
            if high_block:
                yield from wait(empty[s], n - 1)
                pending.append(full[s])    # a copy that lands some time
            else:
                yield from wait(raw_empty[lows % RAW], lows // RAW - 1)
                pending.append(raw_full[lows % RAW])
                lows += 1
            yield

    def expander():
        lows = 0
        for i, high_block in enumerate(blocks):
            if not high_block:
                s, n = i % stages, i // stages
                yield from wait(raw_full[lows % RAW], lows // RAW)
                yield from wait(empty[s], n - 1)
                yield
                full[s].done += 1
                raw_empty[lows % RAW].done += 1
                lows += 1

    def consumer():
        for i in range(len(blocks)):
            s, n = i % stages, i // stages
            yield from wait(full[s], n)
            yield
            empty[s].done += 1

    actors = [producer(), expander(), consumer()]
    weights = [rng.choice((1, 1, 5, 20)) for _ in range(4)]
    for _ in range(4000):
        if not actors or not sound:
            break
        k = rng.choices(range(len(actors) + 1), weights[:len(actors) + 1])[0]
        if k == len(actors):
            if pending:
                pending.pop(0).done += 1
            continue
        try:
            next(actors[k])
        except StopIteration:
            del actors[k]
    return sound and not actors


@pytest.mark.parametrize("stages", [3, 4, 5, 8])
def test_three_stages_and_more_are_sound(stages):
    rng = random.Random(stages)
    for low in range(1, 8):
        for high in range(0, 6):
            for _ in range(10):
                assert run(low, high, 4, stages, rng), (low, high)


def test_two_stages_are_not():
    rng = random.Random(2)
    assert not all(run(2, 2, 4, 2, rng) for _ in range(50))
    assert not all(run(4, 1, 4, 2, rng) for _ in range(50))
