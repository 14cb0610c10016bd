"""The forward point's operators without a GPU: the header's names, its use from C, and what the calls refuse."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward, zo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000  # never dereferenced: validation rejects first
NAN = float("nan")


@pytest.fixture(scope="module")
def L():
    zo_build.build()
    return forward._lib()


def test_exports_every_declared_symbol(L):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "zo_forward.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(zo_[a-z0-9_]+)\s*\(", src)))
    assert set(names) == set(forward.EXPORTS)
    for n in names:
        assert hasattr(L, n), n


def rows(*v):
    return ctypes.addressof(_keep((ctypes.c_int64 * 3)(*v)))


def pages(*v):
    return ctypes.addressof(_keep((ctypes.c_int64 * 4)(*v)))


_kept = []


def _keep(a):
    _kept.append(a)
    return a


def test_rotary_table_validation(L):
    def call(table=FAKE, rows=4, dim=8, base=1e4, scale=1.0, original=0, low=1.0, high=32.0, mag=1.0):
        return L.zo_rotary_table(table, rows, dim, base, scale, original, low, high, mag, None)
    for bad in ({"rows": -1}, {"dim": 7}, {"dim": 0}, {"dim": 258}, {"base": 0.0}, {"base": NAN}, {"scale": 0.0},
                {"scale": NAN}, {"original": -1}, {"low": 33.0}, {"high": NAN}, {"mag": NAN}, {"table": None}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(table=FAKE + 2) == zo.ZO_ERR_ALIGN
    assert call(rows=0, table=None) == zo.ZO_OK


def test_document_spans_validation(L):
    def call(q=FAKE, k=FAKE, prefix=None, docs=2, spans=FAKE, tokens=5):
        return L.zo_document_spans(q, k, prefix, docs, spans, tokens, None)
    for bad in ({"docs": -1}, {"tokens": -1}, {"tokens": 1 << 31}, {"q": None}, {"k": None}, {"spans": None}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(prefix=FAKE + 1) == zo.ZO_ERR_ALIGN
    assert call(tokens=0, spans=None) == zo.ZO_OK


def test_rotate_heads_validation(L):
    def call(part=None, n=1, tokens=3, dim=64, dtype=1, table=FAKE, table_rows=8, rotary=64, layout=0, positions=FAKE,
             slots=None, index=8, n_slots=0, page=1, eps=1e-6):
        p = [FAKE, 128, 64, FAKE + 4096, 0, 128, 64, 0, 2 << 32, 1] if part is None else part
        arr = (ctypes.c_int64 * 10)(*p)
        return L.zo_rotate_heads(ctypes.addressof(arr) if n else None, n, tokens, dim, dtype, table, table_rows, rotary,
                                 layout, positions, slots, index, n_slots, page, eps, None)

    def part(**kw):
        p = dict(i=FAKE, it=128, ih=64, o=FAKE + 4096, op=0, ot=128, oh=64, w=0, wd=0, heads=2, flags=1, reserved=0) | kw
        return [p["i"], p["it"], p["ih"], p["o"], p["op"], p["ot"], p["oh"], p["w"], p["wd"] | p["heads"] << 32,
                p["flags"] | p["reserved"] << 32]
    for bad in ({"n": 4}, {"n": -1}, {"tokens": -1}, {"tokens": 1 << 31}, {"dim": 0}, {"dim": 257}, {"rotary": 63},
                {"rotary": 66}, {"rotary": 0}, {"layout": 2}, {"positions": None}, {"table": None}, {"table_rows": -1},
                {"index": 2}, {"eps": -1.0}, {"eps": NAN}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    for bad in ({"heads": 0}, {"heads": 1025}, {"flags": 4}, {"reserved": 1}, {"i": 0}, {"o": 0}, {"it": -1}, {"oh": -1},
                {"op": -1}, {"flags": 3}):           # slotted without slots
        assert call(part(**bad)) == zo.ZO_ERR_ARG, bad
    assert call(part(flags=2), slots=FAKE, n_slots=8, page=0) == zo.ZO_ERR_ARG
    assert call(part(flags=2), slots=FAKE, n_slots=-1) == zo.ZO_ERR_ARG
    assert call(dtype=3) == zo.ZO_ERR_DTYPE
    assert call(part(w=FAKE, wd=7)) == zo.ZO_ERR_DTYPE
    assert call(part(i=FAKE + 1)) == zo.ZO_ERR_ALIGN
    assert call(part(w=FAKE + 2, wd=0)) == zo.ZO_ERR_ALIGN
    assert call(positions=FAKE + 4) == zo.ZO_ERR_ALIGN
    assert call(tokens=0) == zo.ZO_OK and call(n=0) == zo.ZO_OK


def test_attention_validation(L):
    def call(q=rows(FAKE, 128, 64), k=rows(FAKE, 64, 64), v=rows(FAKE, 64, 64), out=rows(FAKE, 128, 64), tq=4, tk=4, heads=2,
             kv=1, dim=64, dtype=1, spans=FAKE, scale=1.0, cap=0.0, slopes=None, lse=None):
        return L.zo_attention(q, k, v, out, tq, tk, heads, kv, dim, dtype, spans, scale, cap, slopes, lse, None)
    for bad in ({"q": None}, {"out": None}, {"q": rows(0, 1, 1)}, {"k": rows(0, 1, 1)}, {"v": rows(FAKE, -1, 1)},
                {"tq": -1}, {"tk": -1}, {"tq": 1 << 31}, {"heads": 0}, {"heads": 3, "kv": 2}, {"kv": 0}, {"dim": 0},
                {"dim": 257}, {"heads": 1025}, {"spans": None}, {"scale": NAN}, {"cap": -1.0}, {"cap": NAN}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=-1) == zo.ZO_ERR_DTYPE
    for bad in ({"q": rows(FAKE + 1, 1, 1)}, {"spans": FAKE + 2}, {"slopes": FAKE + 2}, {"lse": FAKE + 1}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(tq=0, spans=None) == zo.ZO_OK


def test_decode_validation(L):
    def call(q=rows(FAKE, 128, 64), k=pages(FAKE, 1024, 64, 64), v=pages(FAKE, 1024, 64, 64), out=rows(FAKE, 128, 64),
             batch=2, heads=2, kv=1, dim=64, dtype=1, table=FAKE, stride=4, most=4, n=9, page=16, lengths=FAKE, scale=1.0,
             cap=0.0, slopes=None, lse=None):
        return L.zo_attention_decode(q, k, v, out, batch, heads, kv, dim, dtype, table, stride, most, n, page, lengths, scale,
                                     cap, slopes, lse, None)
    for bad in ({"q": None}, {"k": None}, {"k": pages(0, 1, 1, 1)}, {"v": pages(FAKE, 1, -1, 1)}, {"out": rows(0, 1, 1)},
                {"batch": -1}, {"batch": 1 << 30}, {"heads": 3, "kv": 2}, {"dim": 300}, {"table": None}, {"stride": -1},
                {"most": -1}, {"n": -1}, {"most": 1 << 31}, {"page": 0}, {"lengths": None}, {"scale": float("inf")}, {"cap": -2.0}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=5) == zo.ZO_ERR_DTYPE
    for bad in ({"k": pages(FAKE + 1, 1, 1, 1)}, {"table": FAKE + 1}, {"lengths": FAKE + 2}, {"lse": FAKE + 2}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(batch=0, lengths=None) == zo.ZO_OK


def test_token_loss_validation(L):
    ws = L.zo_token_loss_workspace_size(10)
    assert ws == 80 and L.zo_token_loss_workspace_size(0) > 0

    def call(logits=FAKE, row=100, tokens=10, vocab=100, dtype=1, targets=FAKE, tb=8, flags=0, loss=FAKE, nll=None, w=FAKE, wb=ws):
        return L.zo_token_loss(logits, row, tokens, vocab, dtype, targets, tb, flags, loss, nll, w, wb, None)
    for bad in ({"tokens": -1}, {"tokens": 1 << 29}, {"vocab": 0}, {"vocab": 1 << 31}, {"row": -1}, {"tb": 2}, {"flags": 8},
                {"loss": None}, {"logits": None}, {"targets": None}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=3) == zo.ZO_ERR_DTYPE
    for bad in ({"logits": FAKE + 1}, {"targets": FAKE + 4}, {"loss": FAKE + 4}, {"nll": FAKE + 2}, {"w": FAKE + 4}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(w=None) == zo.ZO_ERR_WORKSPACE and call(wb=ws - 1) == zo.ZO_ERR_WORKSPACE


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 2, 8)
    i = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        forward.rotate_heads(x, table=x[0], positions=i)
    with pytest.raises(TypeError):
        forward.attention(x, x, x, i)
    with pytest.raises(TypeError):
        forward.decode_attention(x, x[None], x[None], i, i)
    with pytest.raises(TypeError):
        forward.token_loss(x[0], i)
    with pytest.raises(ValueError):
        forward.rotary_table(4, 8, device="cpu")


def test_header_is_plain_c_and_links_from_c(tmp_path, L):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    src = tmp_path / "use_forward.c"
    src.write_text(
        "#include <stdio.h>\n#include \"zo_forward.h\"\n"
        "int main(void) {\n"
        "  zo_rows r = {0, 0, 0};\n  zo_head_part p = {{0, 0, 0}, {0, 0, 0, 0}, 0, ZO_BF16, 1, ZO_HEADS_ROTATE, 0};\n"
        "  if (sizeof(p) != 80 || sizeof(zo_pages) != 32) return 1;\n"
        "  if (zo_attention(&r, &r, &r, &r, -1, 0, 1, 1, 64, ZO_BF16, NULL, 1.0f, 0.0f, NULL, NULL, NULL) != ZO_ERR_ARG) return 2;\n"
        "  if (zo_rotate_heads(&p, 1, 0, 64, ZO_BF16, NULL, 0, 64, ZO_ROTARY_HALF, NULL, NULL, 8, 0, 1, 1e-6f, NULL) != ZO_OK)\n"
        "    return 3;\n"
        "  if (zo_token_loss_workspace_size(3) != 24) return 4;\n"
        "  puts(\"ok\");\n  return 0;\n}\n")
    exe = tmp_path / "use_forward"
    lib = zo.LIB_PATH
    r = subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                        str(exe), "-L", os.path.dirname(lib), "-l:" + os.path.basename(lib),
                        "-Wl,-rpath," + os.path.dirname(lib)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stdout, r.stderr)
