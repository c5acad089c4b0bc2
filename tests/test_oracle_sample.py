"""The oracles of eb_sample and eb_kv_assign, pinned by cases worked out by hand."""
import math

import numpy as np
import pytest

from oracle.assign import assign
from oracle.sample import kept_ids, sample

LOG = math.log
Z = [LOG(1), LOG(4), LOG(2), LOG(4), LOG(5)]           # weights 1 4 2 4 5 of 16; order 4 1 3 2 0


@pytest.mark.parametrize("kw,kept", [
    (dict(), [0, 1, 2, 3, 4]),
    (dict(top_k=1), [4]),
    (dict(top_k=2), [1, 4]),                           # of two equal logits the lower id
    (dict(top_k=3), [1, 3, 4]),
    (dict(top_k=7), [0, 1, 2, 3, 4]),
    (dict(top_p=0.0), [4]),
    (dict(top_p=0.3), [4]),                            # 5 >= 4.8
    (dict(top_p=0.32), [1, 4]),                        # 5 < 5.12
    (dict(top_p=0.6), [1, 3, 4]),
    (dict(top_p=0.9), [1, 2, 3, 4]),
    (dict(top_k=3, top_p=0.7), [1, 3, 4]),             # of 13: 9 < 9.1
    (dict(top_k=3, top_p=0.69), [1, 4]),               # 9 >= 8.97
    (dict(min_p=0.5), [1, 3, 4]),
    (dict(min_p=0.79), [1, 3, 4]),
    (dict(min_p=0.81), [4]),
    (dict(min_p=1.0), [4]),
    (dict(temperature=0.0), [4]),
    (dict(temperature=0.5, min_p=0.5), [1, 3, 4]),     # squares: 16/25
    (dict(temperature=0.5, min_p=0.65), [4]),
])
def test_kept(kw, kept):
    assert kept_ids(Z, **kw)[0].tolist() == kept


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.0624, 0), (0.0626, 1), (0.312, 1), (0.313, 2),
                                     (0.437, 2), (0.438, 3), (0.687, 3), (0.688, 4), (0.9999, 4)])
def test_drawn(u, token):
    got = sample(Z, u)
    assert got[0] == token
    assert got[1] == pytest.approx([1, 4, 2, 4, 5][token] / 16, rel=1e-12)
    assert got[2] == pytest.approx(got[1], rel=1e-12)


def test_drawn_on_the_border():
    z = [0.0] * 8
    assert [sample(z, i / 8)[0] for i in range(8)] == list(range(8))
    assert sample([-np.inf, 0.0, -np.inf, 0.0], 0.0)[0] == 1
    assert sample([-np.inf, 0.0, -np.inf, 0.0], 0.5)[0] == 3


def test_rows_without_a_token():
    assert sample([-np.inf] * 3, 0.5) == (-1, 0.0, 0.0)
    assert sample([0.0, np.nan], 0.5)[0] == -1 and math.isnan(sample([0.0, np.nan], 0.5)[1])
    assert sample([0.0, np.inf], 0.5)[0] == -1


def test_confidence_is_the_models():
    token, prob, conf = sample(Z, 0.99, temperature=0.5, top_k=2)
    assert (token, prob, conf) == (4, pytest.approx(25 / 41), pytest.approx(5 / 16))


def test_pages_by_hand():
    table = np.array([[7, 9, 9], [3, 9, 9], [5, 6, 9], [8, 9, 9]], np.int32)
    ring = np.array([20, 21, 0, 0, 0, 0, 0, 0, 0, 22], np.int32)     # free: 22, 20, 21
    got = assign(table, ring, [9, 3], [16, 3, 20, 15], [17, 2, 0, 1], 16, 22, done=[0, 0, 1, 0])
    # two pages, spare rows of the held page, a finished one, the held page's last row
    assert got["table"].tolist() == [[7, 22, 20], [3, 9, 9], [5, 6, 9], [8, 9, 9]]
    assert got["ring"].tolist() == [20, 21, 5, 6, 0, 0, 0, 0, 0, 22]
    assert got["state"].tolist() == [1, 3]
    assert got["cu_block"].tolist() == [0, 17, 19, 19, 20]
    assert got["cu_prefix"].tolist() == [0, 16, 19, 19, 34]
    assert got["pos"].tolist() == list(range(16, 33)) + [3, 4, 15, -1, -1]
    # (n_pages is 10 here: numbers from 10 on are no page)
    assert got["slot"].tolist() == [-1] * 17 + [3 * 16 + 3, 3 * 16 + 4, 8 * 16 + 15, -1, -1]
    assert got["short"].tolist() == [0, 0, 0, 0]


def test_pages_run_out():
    table = np.full((4, 2), 4, np.int32)
    ring = np.arange(8, dtype=np.int32)
    got = assign(table, ring, [6, 2], [0, 0, 5, 16], [16, 32, 3, 16], 16, 80)
    # one page; two where one is left; none needed; one, counted behind the refused two
    assert got["short"].tolist() == [0, 1, 0, 1]
    assert got["table"].tolist() == [[6, 4], [-1, -1], [4, 4], [4, -1]]
    assert got["state"].tolist() == [7, 1]
    assert got["pos"].tolist() == list(range(16)) + [-1] * 32 + [5, 6, 7] + [-1] * 29


def test_pages_wide_and_shared():
    table = np.arange(8, dtype=np.int32).reshape(2, 4)
    ring = np.zeros(8, np.int32)
    got = assign(table, ring, [0, 0], [64, 60], [1, 9], 16, 1, done=[0, 1], shared=[9, 3])
    assert got["short"].tolist() == [1, 0] and got["table"].tolist() == table.tolist()
    assert got["ring"].tolist() == [7] + [0] * 7 and got["state"].tolist() == [0, 1]
