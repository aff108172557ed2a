"""Prompts and chunks behind a window whose keys are cut into parts, against the oracle."""
import numpy as np
import pytest

from answer_util import Round, attention_descs, attention_job, check_attention
from oracle import answer
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu
INF, MINUS, NAN = 0x7f80, 0xff80, 0x7fc0


def run(jobs, in_parts=True):
    r = Round([(p, l) for p, l, _ in jobs])
    descs, keep = attention_descs(r, jobs)
    was = r.dp.pool.stats()["gemm_launches"]
    assert r.dp.pool.grouped_attention(descs, stream=r.dp.stream) == salus.OK, r.dp.pool.last_error()
    r.dp.sync()
    # a launch for each width, and one that joins parts
    assert r.dp.pool.stats()["gemm_launches"] - was == len({s["D"] for _, _, s in jobs}) + in_parts
    check_attention(r, jobs)
    r.check_rest("y", "work")
    r.close()


# new rows and lengths of the sequences, query heads of the key head, window
CASES = [([(80, 2500)], 2, 1000), ([(130, 3000), (90, 90), (70, 2000)], 3, 1500), ([(300, 6000)], 1, 2999), ([(200, 4100), (1, 4100), (0, 50), (65, 1025)], 7, 1025),
         ([(64, 5000), (64, 4000)], 1, 4096), ([(257, 1300), (257, 2800)], 4, 1280)]


@pytest.mark.parametrize("number", range(len(CASES)))
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
def test_windows_of_several_parts(D, number):
    seqs, G, window = CASES[number]
    rng = np.random.default_rng(D + number)
    run([attention_job(rng, seqs, G * (1 + number % 2), 1 + number % 2, D, 32 << number % 3, window, gap=number % 3, tail=number % 2)])


@pytest.mark.parametrize("limit", [2500, 2600, 9000, 100000])
@pytest.mark.parametrize("D", [64, 192])
def test_bounds_above_the_lengths(D, limit):
    """Parts by the window's span, or by the bound where that leaves room for fewer; tiles with fewer parts than others."""
    rng = np.random.default_rng(limit)
    run([attention_job(rng, [(100, 2500), (70, 1300), (90, 90)], 2, 1, D, 64, 1700, max_len=limit, max_pages=-(-limit // 64))])


def spoiled(rng, n, length, window, D, tokens, which, bits):
    p, l, sizes = attention_job(rng, [(n, length)], 2, 1, D, 32, window)
    for i, t in enumerate(tokens):
        at = int(l["table"][0, t // 32]), 0, t % 32
        if which == "k":
            p["k"][answer.key_at(*at, np.arange(D), 1, 32, D)] = bits
        else:
            p["v"][answer.value_at(*at, (5 + 7 * i) % D, 1, 32, D)] = bits
    return p, l, sizes


@pytest.mark.parametrize("bits", [INF, MINUS, NAN])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("n,length,window", [(100, 3000, 1500), (70, 2570, 1100)])
def test_what_is_no_number_at_the_ends_of_a_window(n, length, window, D, which, bits):
    """The last token that no row sees, the first that one sees, one seen by half of the rows, the first that all see; the same at the rows themselves."""
    first = length - n
    back = [first - window, first - window + 1, first - window + n // 2, length - window]
    front = [first, first + 1, first + n // 2, length - 1]
    for tokens in (back[:1], back[1:2], back, front[-2:]) if which == "k" else (back, front, back + front):
        run([spoiled(np.random.default_rng(n), n, length, window, D, tokens, which, bits)])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_missing_pages_in_a_window(D):
    p, l, sizes = attention_job(np.random.default_rng(D), [(90, 3000), (80, 2400)], 2, 1, D, 32, 1400)
    l["table"][0, [44, 45, 60, 93]] = -1                     # at the window's beginning, inside, at its end
    l["table"][1, 20:60] = sizes["n_pages"]                  # whole parts
    run([(p, l, sizes)])


def test_jobs_of_all_widths_together():
    rng = np.random.default_rng(9)
    run([attention_job(rng, [(64 + 20 * j, 1500 + 300 * j)], 2, 1 + j % 2, D, 32, 1100 + 100 * j) for j, D in enumerate((32, 64, 96, 128, 192, 256))])
