"""Mutation check of the attention oracle's pins (tests/test_oracle_attention*.py):
as tests/test_oracle_mutants.py, whose staging it uses, for oracle/attention.py.
Each mutant lives in a temporary copy, on the CPU; its pins must fail."""

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_oracle_mutants import ROOT, _stage

F = "attention.py"

# (name, text, replacement); the text occurs exactly once in oracle/attention.py.
MUTANTS = [
    ("mean_is_sum", "mean = np.mean(y * y, axis=2, keepdims=True)", "mean = np.sum(y * y, axis=2, keepdims=True)"),
    ("eps_outside_sqrt", "np.sqrt(mean + float(np.float32(eps)))", "(np.sqrt(mean) + float(np.float32(eps)))"),
    ("gamma_dropped", "np.sqrt(mean + float(np.float32(eps))) * gamma", "np.sqrt(mean + float(np.float32(eps)))"),
    ("pairs_by_the_other_order", "(2 * i, 2 * i + 1) if interleaved else", "(2 * i, 2 * i + 1) if not interleaved else"),
    ("turned_backwards", "y[:, :, a] * np.cos(angle) - y[:, :, b] * np.sin(angle)",
     "y[:, :, a] * np.cos(angle) + y[:, :, b] * np.sin(angle)"),
    ("second_of_a_pair_unturned", "y[:, :, b] * np.cos(angle) + y[:, :, a] * np.sin(angle)", "y[:, :, b] * np.cos(angle)"),
    ("angle_in_frequency_order", "float(np.float32(inv_freq[i]))", "float(np.float32(inv_freq[half - 1 - i]))"),
    ("sign_of_zero_lost", "np.where(np.signbit(x) & ~np.isnan(x), mag | 128, mag)", "np.where(x < 0, mag | 128, mag)"),
    ("scale_strict", "while amax > E4M3_MAX * s:", "while amax >= E4M3_MAX * s:"),
    ("scale_for_240", "while amax > E4M3_MAX * s:", "while amax > 240.0 * s:"),
    ("scale_floor", "SCALE_FLOOR = 2.0 ** -100", "SCALE_FLOOR = 2.0 ** -90"),
    ("keys_element_order", "inside = (e // 16) * 256 + u * 16 + e % 16", "inside = u * dim + e"),
    ("values_token_order", "(u // 4) * 256 + (e % 16) * 16 + (e // 16 % 4) * 4 + u % 4",
     "(u // 4) * 256 + (e % 16) * 16 + u % 4 * 4 + e // 16 % 4"),
    ("codes_of_the_other_kind", "self.codes = [np.array(k), np.array(v)]", "self.codes = [np.array(v), np.array(k)]"),
    ("scales_of_the_other_kind", "np.array(k_scale, dtype=np.float64), np.array(v_scale, dtype=np.float64)]",
     "np.array(v_scale, dtype=np.float64), np.array(k_scale, dtype=np.float64)]"),
    ("tokens_below_0_kept", "if 0 <= t < table.shape[1] * self.page_size:",
     "if t < table.shape[1] * self.page_size:"),
    ("rows_of_the_next_sequence", "            row += n\n            for entry",
     "            row += max(n, 1) - 1\n            for entry"),
    ("scale_never_grows", "s = max(s, held)", "s = held"),
    ("scale_forgets_held", "s = max(s, held)", "s = s"),
    ("held_codes_left", "* (held / s)", "* 1.0"),
    ("held_codes_the_wrong_way", "* (held / s)", "* (s / held)"),
    ("held_slots_one_more", "self.codes[kind][page, h, :slots[0]] = e4m3_codes(old)",
     "self.codes[kind][page, h, 1:slots[0] + 1] = e4m3_codes(old)"),
    ("page_never_anew", "if slots[0] > 0:", "if True:"),
    ("static_scale_set", "if not static:", "if True:"),
    ("scale_of_page_0", "* self.scale[kind][page, head]", "* self.scale[kind][0, head]"),
    ("page_outside_is_zero", "if 0 <= page < self.pages:\n                x[t]",
     "there[t] = True\n            if 0 <= page < self.pages:\n                x[t]"),
    ("heads_interleaved", "k, there = cache.sequence(0, table[b], h // group, length)",
     "k, there = cache.sequence(0, table[b], h % cache.heads, length)"),
    ("row_is_its_place", "t = max(int(kv_len[b]), 0) - n + i", "t = i"),
    ("causal_strict", "(j <= t) if causal", "(j < t) if causal"),
    ("window_one_more", "(j > t - window)", "(j >= t - window)"),
    ("window_ignores_causal", "(j > t - window) if window > 0 else True",
     "(j > length - 1 - window) if window > 0 else True"),
    ("scale_dropped", "s = k[seen] @ q[row + i, h] * scale", "s = k[seen] @ q[row + i, h]"),
    ("not_normalized", "w @ v[seen] / w.sum()", "w @ v[seen]"),
    ("lse_without_maximum", "s.max() + np.log(w.sum())", "np.log(w.sum())"),
    ("bound_signed_values", "w @ np.abs(v[seen]) / w.sum()", "w @ v[seen] / w.sum()"),
    ("bound_signed_scores", "(np.abs(k[seen]) @ np.abs(q[row + i, h])).max() * abs(scale)",
     "(k[seen] @ q[row + i, h]).max() * abs(scale)"),
    ("bound_of_one_token", "len(held) * E4M3_MAX * max(held)", "E4M3_MAX * max(held)"),
]


def _pins_pass(mutant):
    tmp = tempfile.mkdtemp(prefix="oracle_mutant_")
    try:
        _stage(tmp, None if mutant is None else (mutant[0], F) + mutant[1:])
        r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                            "tests/test_oracle_attention.py", "tests/test_oracle_attention_cache.py"], cwd=tmp,
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
