"""CPU-only checks of the losses' C entries: every declared symbol is exported and marshalled, the argument structs have
the header's layout, and bad arguments are refused before anything touches a GPU."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest

from paper_1901_01544_b200 import binding, build, losses

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "iwp_loss.h")
E = binding.IWP_ERR_INVALID


@pytest.fixture(scope="module")
def L():
    build.build()
    return losses.lib()


def test_header_and_library_agree(L):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(iwp_[a-z_0-9]+)\s*\(", src)))
    assert names == sorted(losses.EXPORTS)
    for n in names:
        assert hasattr(L, n)


def test_structs_have_the_headers_layout(tmp_path):
    fields = {"iwp_head_args": losses.HeadArgs, "iwp_balance_args": losses.BalanceArgs}
    lines = ['#include "%s"' % HEADER, "#include <cstddef>", "#include <cstdio>", "int main() {"]
    for name, cls in fields.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        for f, _ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, f))
    (tmp_path / "l.cpp").write_text("\n".join(lines + ["}"]))
    subprocess.run(["g++", str(tmp_path / "l.cpp"), "-o", str(tmp_path / "l")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls in fields.values():
        want += [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def head(**kw):
    a = losses.HeadArgs(tokens=8, vocab=100, dim=64, dtype=1, hidden=256, hidden_ld=64, weight=256, weight_ld=64, targets=256, top_k=1,
                        lse=256, temperature=1.0, scale=1.0, dhidden=256, dhidden_ld=64, dhidden_type=1, dweight=256, dweight_ld=64,
                        dweight_type=0, workspace=256, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(vocab=0), dict(dim=0), dict(tokens=1 << 31), dict(dtype=0), dict(dtype=3), dict(hidden=None), dict(weight=None),
    dict(lse=None), dict(hidden_ld=63), dict(weight_ld=63), dict(dhidden_ld=63), dict(dweight_ld=63), dict(dhidden_type=2),
    dict(dweight_type=7), dict(workspace=None), dict(workspace=257), dict(hidden=257), dict(dweight=258, dweight_type=0),
    dict(scale=math.nan), dict(scale=math.inf), dict(piece_bytes=-1), dict(have_lse=1, dhidden=None, dweight=None),
    dict(targets=None, top_ids=None), dict(targets=None, top_ids=256, top_ids_ld=1, ids_bytes=8),
    dict(targets=None, top_k=0), dict(targets=None, top_k=1025),
    dict(targets=None, top_ids=256, top_ids_ld=1, ids_bytes=2, top_logits=256, top_logits_ld=1),
    dict(targets=None, top_ids=256, top_ids_ld=1, ids_bytes=4, top_logits=256, top_logits_ld=1, top_type=5),
    dict(targets=None, top_ids=256, top_ids_ld=1, ids_bytes=4, top_logits=256, top_logits_ld=1, temperature=0.0),
    dict(targets=None, top_ids=256, top_ids_ld=1, ids_bytes=4, top_logits=256, top_logits_ld=1, temperature=math.inf),
])
def test_head_refuses(L, bad):
    assert L.iwp_head_loss(C.byref(head(**bad)), None) == E


def test_head_workspace(L):
    need = L.iwp_head_workspace(C.byref(head()))
    assert need > 0
    assert L.iwp_head_workspace(C.byref(head(vocab=0))) == -1 and L.iwp_head_workspace(None) == -1
    assert L.iwp_head_loss(C.byref(head(workspace_bytes=need - 1)), None) == binding.IWP_ERR_CAPACITY
    assert L.iwp_head_loss(None, None) == E
    # the workspace never shrinks when tokens grow, and the probabilities of a piece are bounded
    last = 0
    for T in (1, 7, 128, 129, 1000, 4096, 8192, 30000):
        n = L.iwp_head_workspace(C.byref(head(tokens=T, vocab=131072, dim=4096, hidden_ld=4096, weight_ld=4096, dhidden_ld=4096, dweight_ld=4096)))
        assert n >= last
        last = n
    small = L.iwp_head_workspace(C.byref(head(tokens=4096, vocab=131072, piece_bytes=1 << 24)))
    whole = L.iwp_head_workspace(C.byref(head(tokens=4096, vocab=131072, piece_bytes=1 << 34)))
    assert small < 1 << 27 and whole > 2 * 4096 * 131072
    # operands whose rows do not start at multiples of 16 bytes need room for copies
    assert L.iwp_head_workspace(C.byref(head(hidden_ld=65))) > need and L.iwp_head_workspace(C.byref(head(weight=258))) > need


def balance(**kw):
    a = losses.BalanceArgs(tokens=8, experts=16, top_k=2, type=0, ids_bytes=8, logits=256, logits_ld=16, ids=256, ids_ld=2, counts=256,
                           dlogits=256, dlogits_ld=16, workspace=256, workspace_bytes=1 << 40, coef=1.0, scale=1.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(tokens=-1), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=17), dict(type=3), dict(logits=None), dict(ids=None),
    dict(counts=None), dict(workspace=None), dict(workspace=128), dict(logits_ld=15), dict(ids_ld=1), dict(ids_bytes=3), dict(dlogits_ld=15),
    dict(logits=258), dict(ids=260), dict(dlogits=258), dict(coef=math.nan), dict(scale=math.inf),
])
def test_balance_refuses(L, bad):
    assert L.iwp_balance_loss(C.byref(balance(**bad)), None) == E


def test_balance_workspace(L):
    need = L.iwp_balance_workspace(C.byref(balance()))
    assert need > 0 and L.iwp_balance_workspace(C.byref(balance(experts=0))) == -1
    assert L.iwp_balance_loss(C.byref(balance(workspace_bytes=need - 1)), None) == binding.IWP_ERR_CAPACITY
    assert L.iwp_loss_reset(None, None) == E and L.iwp_loss_status(None, None, None) == E
