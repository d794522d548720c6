"""The ring by which the experts' kernels load, as a model on the CPU: no order in which loaders and reader take their steps lets a
stage be written while it is in use.  The model's constants and rule are those of the source."""
import os
import random
import re

import pytest

import ring_model

SOURCE = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36301_b200", "csrc",
                           "more_experts_sm100.cu")).read()


def constant(name):
    return eval(re.search(r"constexpr int [^;]*\b%s = ([\d* ]+)[,;]" % name, SOURCE).group(1))


def test_the_model_is_the_source_s():
    assert constant("kSlots") == ring_model.SLOTS and constant("kXRing") == ring_model.RING
    rule = re.search(r"bool wait_empty\([^)]*\)\s*\{(.*?)\n    \}", SOURCE, re.S)
    assert rule, "a phase may be taken for another one of the same parity"
    lines = [x.split("//")[0].strip() for x in rule.group(1).strip().split("\n")]
    assert lines == ["if (last < 0) return true;", "if (last - kSlots > empty && !wait_for(stage - kSlots, c, abort_flag, status)) return false;",
                     "empty = last;", "return wait_for(last, c, abort_flag, status);"]
    # nothing else waits for a stage to be empty, and both kinds of loaders do it that way
    assert len(re.findall(r"mbar_wait\w*\(smem_u32\(&\w+->empty\[", SOURCE)) == 1
    assert len(re.findall(r"\bwait_empty\((?:n|own\.stage), (?:own\.)?last, ", SOURCE)) == 2


@pytest.mark.parametrize("which,loaders", [(0, "kTeams"), (1, "kFewLoaders"), (2, "kBackLoaders"), (3, "kBackLoaders")])
def test_no_stage_is_written_while_it_is_in_use(which, loaders):
    lengths = ring_model.kinds()[which]
    for seed in range(80):
        rng = random.Random(seed)
        assert ring_model.run(ring_model.sequence(rng, lengths), constant(loaders), rng, "own slot", rng.choice([0.0, 0.2, 0.5, 0.9])), seed


def test_the_model_sees_what_goes_wrong_by_parity_alone():
    """Without the wait in front a phase is taken for done; with one for the wrong stage it is missed."""
    lengths = ring_model.kinds()[3]
    for rule, right in ((None, False), ("same slot", False), ("own slot", True)):
        results = []
        for seed in range(40):
            rng = random.Random(seed)
            results.append(ring_model.run(ring_model.sequence(rng, lengths), 7, rng, rule, rng.choice([0.0, 0.2, 0.5, 0.9])))
        assert all(results) == right, rule
