"""The oracle of answering models against worked examples and other formulations."""
import numpy as np
import torch

from oracle import answer
from paper_1902_04610_amd import synth


def bits(a):
    return synth.f32_to_bf16_bits(np.ascontiguousarray(a, np.float32))


def test_places_in_the_cache_are_a_permutation():
    Hkv, page, D, n = 2, 64, 32, 3
    for at in (answer.key_at, answer.value_at):
        places = {at(p, h, t, d, Hkv, page, D) for p in range(n) for h in range(Hkv) for t in range(page) for d in range(D)}
        assert places == set(range(n * Hkv * page * D))
        assert at(1, 0, 0, 0, Hkv, page, D) == Hkv * page * D and at(0, 1, 0, 0, Hkv, page, D) == page * D


def test_rotation_by_hand():
    head = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(answer.rotate(head, 1, [np.pi / 2], 0, 1.0)[0], [-2, 1, 3, 4])
    assert np.allclose(answer.rotate(head, 1, [np.pi / 2, np.pi], 0, 1.0)[0], [-3, -2, 1, -4])
    assert np.allclose(answer.rotate(head, 1, [np.pi / 2, np.pi], 1, 2.0)[0], [-4, 2, -6, -8])


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    a, b, f = rng.standard_normal(16), rng.standard_normal(16), [1.0, 0.3, 0.1, 0.01]
    one = answer.rotate(a, 7, f, 0, 1.0)[0] @ answer.rotate(b, 3, f, 0, 1.0)[0]
    assert np.isclose(one, answer.rotate(a, 1007, f, 0, 1.0)[0] @ answer.rotate(b, 1003, f, 0, 1.0)[0])


def test_attention_of_a_whole_prompt_is_the_textbooks():
    rng = np.random.default_rng(1)
    n, Hq, Hkv, D, page = 40, 4, 2, 32, 32
    q, k, v = (rng.standard_normal((n, h, D)) for h in (Hq, Hkv, Hkv))
    table = np.array([[2, 0]])
    kc, vc = np.zeros(3 * Hkv * page * D, np.uint16), np.zeros(3 * Hkv * page * D, np.uint16)
    d = np.arange(D)
    for t in range(n):
        for h in range(Hkv):
            kc[answer.key_at(table[0, t // page], h, t % page, d, Hkv, page, D)] = bits(k[t, h])
            vc[answer.value_at(table[0, t // page], h, t % page, d, Hkv, page, D)] = bits(v[t, h])
    for window in (0, 5):
        got = answer.attention(bits(q), kc, vc, [0, n], [n], table, n, Hq, Hkv, D, page, 3, window, 0.2, 1000)
        r = lambda a: torch.from_numpy(answer.bf16_values(bits(a))).transpose(0, 1)
        seen = torch.ones(n, n).tril().bool() & (torch.ones(n, n).triu(1 - window).bool() if window else torch.ones(n, n).bool())
        score = (r(q) @ r(k).repeat_interleave(Hq // Hkv, 0).mT * 0.2).masked_fill(~seen, -torch.inf)
        want = (torch.softmax(score, -1) @ r(v).repeat_interleave(Hq // Hkv, 0)).transpose(0, 1).reshape(n, -1)
        assert np.allclose(np.stack([got[i][0] for i in range(n)]), want.numpy())


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    s = lambda u, T=1.0, k=0, p=1.0, m=0.0: answer.sample(x, T, k, p, m, u)
    assert [s(u) for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [s(u, k=2) for u in (0.1, 0.57, 0.58, 0.9)] == [1, 1, 3, 3]
    assert {s(u, p=0.69) for u in np.linspace(0, 0.99, 40)} == {1, 3} and {s(u, p=0.71) for u in np.linspace(0, 0.99, 40)} == {1, 2, 3}
    assert {s(u, m=0.6) for u in np.linspace(0, 0.99, 40)} == {1, 3}
    assert {s(u, k=3, p=0.7, m=0.8) for u in np.linspace(0, 0.99, 40)} == {1}       # 0.4 + 0.3 of 0.9 reach 0.7; 0.3 / 0.4 < 0.8
    assert s(0.9, T=0.0) == 1 and answer.sample(np.array([2.0, 5.0, 5.0]), 0.0, 0, 1.0, 0.0, 0.5) == 1
    assert answer.sample(np.array([np.nan, -np.inf]), 1.0, 0, 1.0, 0.0, 0.5) == -1
    assert [answer.sample(np.zeros(4), 1.0, 2, 1.0, 0.0, u) for u in (0.1, 0.6)] == [0, 1]
