"""The reference of tests/kv_helpers.py against the one of tests/attention_helpers.py where a
step has a row for every token, and by its own rules where it has not."""
import numpy as np
import pytest

from tests import attention_helpers as A
from tests import kv_helpers as K


def _lens(rng, batch):
    return [(int(rng.integers(0, 70)), int(rng.integers(0, 40) if rng.random() < 0.6 else 0)) for _ in range(batch)]


@pytest.mark.parametrize("seed", range(40))
def test_references_agree_where_rows_suffice(seed):
    rng = np.random.default_rng(seed)
    lens = _lens(rng, int(rng.integers(1, 9)))
    c = K.extend_case(lens, 16, seed, stride=int(rng.integers(1, 8)), rows=sum(a for _, a in lens) + seed % 3,
                      n_free=int(rng.integers(0, 9)) if seed % 2 else None)
    a, b = A.extend_ref(**_args(c)), K.extend_ref(**_args(c))
    for name in a:
        assert np.array_equal(a[name], b[name]), name


def _args(c):
    return dict(table=c["table"], cached=c["cached"], added=c["added"], free_pages=c["free"], n_free=c["n_free"],
                page=c["page"], pages=c["pages"], rows=c["rows"])


@pytest.mark.parametrize("seed", range(40))
def test_fewer_rows_than_tokens(seed):
    """Pages are held by a table or on the stack, never neither; and a step of fewer rows is
    a step of fewer tokens."""
    rng = np.random.default_rng(100 + seed)
    lens = _lens(rng, int(rng.integers(1, 9)))
    tokens = sum(a for _, a in lens)
    c = K.extend_case(lens, 16, seed, rows=int(rng.integers(0, tokens + 1)))
    out = K.extend_ref(**_args(c))
    stack = [int(p) for p in c["free"][:out["n_free"][0]]]
    held = [int(out["table"][b, i]) for b in range(len(lens)) for i in range(-(-out["kv_len"][b] // 16))]
    assert len(set(held + stack)) == len(held + stack)
    assert set(held + stack) == {int(p) for p in c["free"]} | {int(p) for p in c["table"].ravel() if p >= 0}
    assert out["short"] == [tokens - c["rows"]]
    fewer = dict(c, added=np.diff(out["q_start"]))
    again = K.extend_ref(**_args(fewer))
    for name in out:
        if name != "short":
            assert np.array_equal(out[name], again[name]), name
