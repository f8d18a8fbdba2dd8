"""When prefill_decode reads in groups: its rule on both sides of what was measured (host arithmetic: this runs without a GPU)."""
import pytest

from paper_2602_00182_amd import decode as dec

CHUNK = 256
# prompts, rows of each, tokens of a prompt, tokens behind it, KV heads; time of an attention call in microseconds, each row for itself and in groups (MI355X)
SLOWER = [(48, 3, 300, 1, 32, 58.6, 79.2), (16, 2, 4100, 4000, 8, 95.0, 119.8), (4, 2, 4100, 4000, 32, 96.0, 119.6), (48, 3, 600, 300, 4, 25.5, 31.4),
          (16, 4, 4100, 4000, 4, 86.2, 102.7), (4, 2, 4100, 300, 16, 26.8, 30.6), (16, 4, 300, 40, 32, 36.3, 41.4), (1, 2, 8200, 40, 16, 19.7, 22.0)]
FASTER = [(4, 16, 4000, 60, 4, 43.0, 21.0), (1, 64, 32000, 500, 8, 427.0, 122.0), (1, 16, 2900, 250, 8, 20.8, 15.8), (6, 10, 2150, 150, 8, 52.0, 28.4),
          (16, 16, 1100, 40, 4, 47.2, 27.3)]


def pays(P, rows, L, tail, Hkv):
    shared = L // CHUNK * CHUNK
    return dec._groups_pay(P, rows, Hkv, P * (rows - 1) * shared, P * rows * (L + tail - shared))


@pytest.mark.parametrize("case", SLOWER)
def test_calls_that_groups_slow_down_are_left_alone(case):
    assert case[6] > case[5] and not pays(*case[:5])


@pytest.mark.parametrize("case", FASTER)
def test_calls_that_gain_most_are_grouped(case):
    assert case[6] < case[5] and pays(*case[:5])


def test_one_row_a_group_never_pays():
    assert not dec._groups_pay(8, 1, 32, 0, 0) and not dec._groups_pay(1, 64, 8, 0, 0)
