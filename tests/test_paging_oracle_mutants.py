"""Mutation check of the paging oracle's pins (tests/test_oracle_paging.py): as
tests/test_oracle_mutants.py, whose staging it uses, for oracle/paging.py.
Each mutant lives in a temporary copy, on the CPU; its pins must fail."""

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_oracle_mutants import ROOT, _stage

F = "paging.py"

# (name, text, replacement); the text occurs exactly once in oracle/paging.py.
MUTANTS = [
    ("pages_rounded_down", "return -(-tokens // self.page)", "return tokens // self.page"),
    ("drop_ignored", "base = max(held - max(drop[b], 0), 0)", "base = held"),
    ("kept_ignored", "self.pages(max(base, min(max(kept[b], 0), held)))", "self.pages(base)"),
    ("nothing_given_back", "self.stack[count] = self.table[b][entry]\n                    count += 1", "count += 0"),
    ("pushed_in_place", "self.stack[count] = self.table[b][entry]", "self.stack[count] = self.stack[count]"),
    ("width_ignored", "if base + want > most:", "if base + want > 10 ** 9:"),
    ("width_strict", "if base + want > most:", "if base + want >= most:"),
    ("page_taken_twice", "entries = range(self.pages(base), self.pages(base + want))",
     "entries = range(base // self.page, self.pages(base + want))"),
    ("pool_strict", "len(taken) + len(entries) > count", "len(taken) + len(entries) >= count"),
    ("pool_ignored", "len(taken) + len(entries) > count", "len(taken) + len(entries) > len(self.stack)"),
    ("rows_ignored", "or cu[-1] + want > rows", "or cu[-1] + want > 10 ** 9"),
    ("later_ones_served", "full = full or len(taken)", "full = len(taken)"),
    ("taken_backwards", "self.stack[self.count + i]", "self.stack[self.count + len(taken) - 1 - i]"),
    ("taken_from_the_front", "self.stack[self.count + i]", "self.stack[i]"),
    ("position_is_its_place", "positions.append(t)", "positions.append(t - self.kv_len[b])"),
    ("slot_of_the_page", "page * self.page + t % self.page if", "page * self.page if"),
    ("bounds_exchanged", "np.stack([hi, lo]) * 127", "np.stack([lo, hi]) * 127"),
    ("top_of_the_largest", "max(np.abs(hi).max(), np.abs(lo).max())", "np.abs(hi).max()"),
    ("bounds_in_128ths", "np.stack([hi, lo]) * 127 / top", "np.stack([hi, lo]) * 128 / top"),
    ("bounds_cut", "np.rint(np.stack([hi, lo]) * 127 / top)", "np.trunc(np.stack([hi, lo]) * 127 / top)"),
    ("scale_dropped", "np.float32(top * float(scale))", "np.float32(top)"),
    ("query_cut", "np.rint(q * 127 / np.where", "np.trunc(q * 127 / np.where"),
    ("unit_dropped", "value = np.float32(float(total) * float(unit))", "value = np.float32(float(total))"),
    ("step_dropped", "return np.float32(float(best) * float(step))", "return np.float32(float(best))"),
    ("smallest_head", "value > best", "value < best"),
    ("largest_only", "np.maximum(i * bounds[0], i * bounds[1])", "(i * bounds[0])"),
    ("all_at_count_strict", "if seen <= count:", "if seen < count - 1:"),
    ("smallest_taken", "else -scores[j], j))", "else scores[j], j))"),
    ("highest_among_equals", "else -scores[j], j))", "else -scores[j], -j))"),
    ("outside_first", "(scores[j] is None, 0 if", "(scores[j] is not None, 0 if"),
    ("first_dropped", "middle = range(first, seen - recent)", "middle = range(0, seen - recent)"),
    ("largest_with_nan", "np.fmax.reduce(values)", "np.maximum.reduce(values)"),
    ("smallest_with_nan", "np.fmin.reduce(values)", "np.minimum.reduce(values)"),
    ("nothing_stays_nan", "np.nan_to_num(np.fmax.reduce(values))", "np.fmax.reduce(values)"),
    ("finite_ignored", "whole = np.isfinite(q).all(axis=1)", "whole = np.ones(len(q), dtype=bool)"),
    ("one_finite_is_enough", "np.isfinite(q).all(axis=1)", "np.isfinite(q).any(axis=1)"),
    ("infinity_left_in", "np.isfinite(q)", "~np.isnan(q)"),
    ("nan_is_largest", "else -np.inf for s in scores", "else np.inf for s in scores"),
    ("nan_is_not_there", "else -np.inf for s in scores", "else None for s in scores"),
    ("recent_dropped", "list(range(seen - recent, seen))", "list(range(seen - 1, seen))"),
]


def _pins_pass(mutant):
    tmp = tempfile.mkdtemp(prefix="oracle_mutant_")
    try:
        _stage(tmp, None if mutant is None else (mutant[0], F) + mutant[1:])
        r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                            "tests/test_oracle_paging.py"], cwd=tmp,
                           env=dict(os.environ, PYTHONDONTWRITEBYTECODE="1"), stdout=subprocess.PIPE,
                           stderr=subprocess.STDOUT, timeout=600)
        return r.returncode == 0, r.stdout.decode(errors="replace")[-2000:]
    finally:
        shutil.rmtree(tmp, ignore_errors=True)


@pytest.mark.parametrize("mutant", MUTANTS, ids=lambda m: m[0])
def test_mutant_texts_are_unique(mutant):
    assert open(os.path.join(ROOT, "oracle", F)).read().count(mutant[1]) == 1


def test_every_mutant_fails_a_pin():
    with ThreadPoolExecutor(max_workers=4) as ex:
        control = ex.submit(_pins_pass, None)
        results = list(ex.map(_pins_pass, MUTANTS))
    ok, out = control.result()
    assert ok, "the unmutated oracle copy must pass its pins:\n" + out
    survivors = [m[0] for m, (passed, _) in zip(MUTANTS, results) if passed]
    assert not survivors, "mutants no pin catches: %s" % survivors
