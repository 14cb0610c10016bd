"""Outputs over inputs are refused by the library, as far as strides show them; addresses here are never dereferenced:
validation refuses first."""
import ctypes

import pytest

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward, zo

A = 0x7F0000000000


@pytest.fixture(scope="module")
def L():
    zo_build.build()
    return forward._lib()


def words(*v):
    return (ctypes.c_int64 * len(v))(*v)


def attention(L, out, q=(A, 128, 64), k=(A + (1 << 30), 64, 64), v=(A + (1 << 31), 64, 64), tq=100, tk=100):
    q, k, v, out = (words(*x) for x in (q, k, v, out))
    return L.zo_attention(q, k, v, out, tq, tk, 2, 1, 64, 1, A, 1.0, 0.0, None, None, None)


K, V = A + (1 << 30), A + (1 << 31)


@pytest.mark.parametrize("out", [
    (A, 128, 64),                    # the queries in place
    (A + 2 * 128, 128, 64),          # a row further
    (A + 2 * 64, 256, 128),          # every other head of the queries' memory, as heads of wider rows
    (A, 64, 6400),                   # their memory with heads first
    (A + 2 * 99 * 128, 128, 64),     # the last row alone
    (A - 2 * 99 * 128, 128, 64),     # the first
    (K + 2 * 64 * 50, 128, 64),      # in the middle of the keys
    (V, 4096, 64), (V + 2 * 64 * 99 + 126, 128, 64),
    (A + (1 << 20), 0, 64),          # rows over one another
    (A + (1 << 20), 128, 0),         # heads over one another
    (A + (1 << 20), 128, 63), (A + (1 << 20), 32, 6400),
])
def test_attention(L, out):
    assert attention(L, out) == zo.ZO_ERR_ARG


def test_attention_of_a_fused_projection(L):
    """Rows of 4 heads, the queries the first two: an output over the second and third."""
    assert attention(L, (A + 2 * 64, 256, 64), q=(A, 256, 64)) == zo.ZO_ERR_ARG
    assert attention(L, (A + 2 * 192, 256, 64), q=(A, 256, 64)) == zo.ZO_ERR_ARG   # into the next row's first head


def decode(L, out, q=(A, 128, 64), k=(K, 1024, 64, 64), v=(V, 1024, 64, 64), batch=4, n=9, page=16):
    q, k, v, out = (words(*x) for x in (q, k, v, out))
    return L.zo_attention_decode(q, k, v, out, batch, 2, 1, 64, 1, A, 4, 4, n, page, A, 1.0, 0.0, None, None, None)


@pytest.mark.parametrize("out", [(A + 128, 128, 64), (A, 64, 256), (K, 128, 64), (K + 2 * 1024 * 8 + 2 * 64 * 15, 128, 64),
                                 (V + 2 * 9 * 1024 - 2, 128, 64), (A + (1 << 20), 0, 64)])
def test_decode(L, out):
    assert decode(L, out) == zo.ZO_ERR_ARG


def rotate(L, parts, tokens=100, slots=None, n_slots=0, page=1):
    flat = []
    for p in parts:
        p = dict(i=A, it=128, ih=64, o=A, op=0, ot=128, oh=64, heads=2, flags=1) | p
        flat += [p["i"], p["it"], p["ih"], p["o"], p["op"], p["ot"], p["oh"], 0, p["heads"] << 32, p["flags"]]
    return L.zo_rotate_heads(words(*flat), len(parts), tokens, 64, 1, A, 8, 64, 0, A, slots, 8, n_slots, page, 1e-6, None)


@pytest.mark.parametrize("parts", [
    [{"o": A + 128}], [{"o": A, "ot": 64, "oh": 6400}], [{"o": A + 256}], [{"o": A + (1 << 20), "ot": 0}],
    [{"o": A + (1 << 20), "oh": 0}],
    [{"o": A + (1 << 20)}, {"i": K, "o": A}],                       # the second's output over the first's input
    [{"i": K, "o": V}, {"i": A, "o": V + 128}],                     # outputs over one another
    [{"i": A, "it": 512, "o": K}, {"i": A + 256, "it": 512, "o": A + 128, "ot": 512}],
])
def test_rotate(L, parts):
    assert rotate(L, parts) == zo.ZO_ERR_ARG


def test_rotate_into_a_cache_over_its_input(L):
    cache = {"i": A + 2 * 1024 * 3, "o": A, "op": 1024, "ot": 128, "flags": 3}
    assert rotate(L, [cache], slots=A, n_slots=9 * 8, page=8) == zo.ZO_ERR_ARG
    assert rotate(L, [{"i": K, "o": A, "op": 1024, "ot": 128, "flags": 3}, {"i": V, "o": A, "op": 1024, "ot": 128, "flags": 2}],
                  slots=A, n_slots=9 * 8, page=8) == zo.ZO_ERR_ARG
