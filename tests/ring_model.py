"""A model, on the CPU, of the ring of stages of varying length by which the experts' kernels load (struct Ring in more_experts_sm100.cu):
loaders that take stages in turn, a reader that empties them in order, and one barrier per slot that is known by the parity of its
phase alone.  Agents take steps in any order that a scheduler likes."""
import random

SLOTS, RING = 16, 153 * 1024


def emptied_before(sizes):
    """For every stage the one that has to be empty before it is written (Ring::mine)."""
    head = end = 0
    begun, out = [], []
    for n, b in enumerate(sizes):
        wraps = head + b > RING
        at = 0 if wraps else head
        start = end
        end += b + (RING - head if wraps else 0)
        head = at + b
        old = 0
        for slot in range(SLOTS):
            stages = [m for m in range(max(0, n - SLOTS), n) if m % SLOTS == slot]
            old += not stages or slot == n % SLOTS or end - RING - begun[stages[-1]] > 0
        begun.append(start)
        out.append((at, n - SLOTS + old - 1))
    return out


def run(sizes, loaders, rng, rule, lazy=0.5):
    """True if all stages are emptied, and none is written while one that it overlaps, or its slot's last, is still to be emptied.
    ``rule``: what a loader waits for in front of the stage that has to be empty, where it does not know the one of that slot before to be:
    "own slot" the stage of the new one's slot, "same slot" that one before, None nothing.  ``lazy``: how seldom the reader takes a step;
    the loaders are slow or quick by turns."""
    plan = emptied_before(sizes)
    phases = [0] * SLOTS                                     # completed phases of a slot's "empty" barrier
    issued, emptied = set(), 0                               # stages written; stages emptied, in order
    at = list(range(loaders))                                # a loader's next stage
    sure = [-1] * loaders                                    # the stage up to which it knows them to be empty
    first = [True] * loaders                                 # the wait in front is still to be made
    pace = [0.7] * loaders

    def passes(m):
        """The wait for stage m: the phase m // SLOTS is taken for done where the barrier's parity says so."""
        return phases[m % SLOTS] & 1 != (m // SLOTS) & 1

    for _ in range(400 * len(sizes)):
        if emptied == len(sizes):
            return True
        if emptied in issued and rng.random() >= lazy:
            phases[emptied % SLOTS] += 1
            emptied += 1
        if rng.random() < 0.05:
            pace[rng.randrange(loaders)] = rng.choice([0.01, 0.05, 0.3, 1.0])
        for i in rng.sample(range(loaders), loaders):
            n = at[i]
            if n >= len(sizes) or rng.random() > pace[i]:
                continue
            where, last = plan[n]
            if last >= 0:
                if rule and first[i] and last - SLOTS > sure[i]:
                    if not passes(n - SLOTS if rule == "own slot" else last - SLOTS):
                        continue
                first[i] = False
                if not passes(last):
                    continue
                sure[i] = last
            if max(last, n - SLOTS) >= emptied:
                return False
            for m in range(emptied, n):
                if m in issued and plan[m][0] < where + sizes[n] and where < plan[m][0] + sizes[m]:
                    return False
            issued.add(n)
            at[i], first[i] = n + loaders, True
    return False                                             # (somebody waits for good)


def kinds():
    """Lengths that the kernels' stages have: a multiple of a box's 8 KB per 64 columns and of a row's 128 bytes."""
    forward = [r * 1024 + b * 8192 for r in range(1, 17) for b in (2, 4)]
    rows = [16384 + b * 8192 for b in (1, 2, 4)]
    act = [n for r in range(1, 17) for b in (1, 2) for one in (r * 1024 + b * 8192,) for n in ((one, 2 * one) if one <= 16384 else (one,))]
    weights = [steps * 2048 * boxes for steps in range(1, 5) for boxes in range(2, 7)]
    return forward, rows, act, weights


def sequence(rng, lengths, n=240):
    """Many of one kind, then many of another."""
    out = []
    while len(out) < n:
        out += [rng.choice(lengths)] * rng.randint(1, 60)
    return out[:n]
