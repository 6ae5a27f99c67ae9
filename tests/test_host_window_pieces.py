"""The forward window kernel's tile loop on the host, in the two forms that it has: D = 64
takes each visible 32-key half of a tile by itself, D = 128 the whole tile, where a hidden
half's scores are not computed and the mask alone keeps them out of the row's maximum."""
import os

import pytest

import test_host_window as host

CALLS = """if (!hide0 && !hide1) piece(2, kb);
          else piece(1, hide0 ? kb + 32 : kb);"""
KEPT = "if (keep_) {"
FORMS = {
    64: ("for (int t = 0; t < 2; ++t)\n          if (!(t ? hide1 : hide0)) piece(ic<1>{}, CAREFUL_, stage, 32 * t, kb + 32 * t, false, false);",
         "for (int t = 0; t < 2; ++t)\n            if (!(t ? hide1 : hide0)) piece(1, kb + 32 * t);"),
    128: ("piece(ic<2>{}, CAREFUL_, stage, 0, kb, hide0, hide1);", "piece(2, kb);"),
}
PLANTS = {                                               # one-off mistakes, by the form that they break
    64: [("kb <= qw + 31 - W", "kb < qw + 31 - W"), ("kb + 32 <= qw - W + 1", "kb + 32 <= qw - W + 2")],
    128: [("kb + 32 * NS - 1 > qw", "kb + 32 - 1 > qw"), ("kb <= qw + 31 - W && kb + 32 * NS > sinks", "kb <= qw - 1 - W && kb + 32 * NS > sinks"),
          ("kb + 64 <= qw - W + 1", "kb + 64 <= qw - W + 2")],
}


def program(D, plant=None):
    src = open(os.path.join(host.CSRC, "attn_window.hip")).read()
    kernel, call = FORMS[D]
    assert " ".join(kernel.split()) in " ".join(src.split())          # the form is still the kernel's
    text = host.program()
    for a, b in ((CALLS, call), (KEPT, "if (keep_ && NS == 2 && (t ? hide1 : hide0)) ++bad;\n                  " + KEPT)):
        assert text.count(a) == 1
        text = text.replace(a, b)
    if plant:
        assert plant[0] in text
        text = text.replace(*plant)
    return text


@pytest.mark.parametrize("D", sorted(FORMS))
def test_pieces_are_the_visible_keys(tmp_path, D):
    r = host._run(tmp_path, program(D))
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("D,plant", [(D, p) for D in sorted(PLANTS) for p in PLANTS[D]])
def test_planted_mistakes_are_found(tmp_path, D, plant):
    r = host._run(tmp_path, program(D, plant))
    assert r.returncode != 0, r.stdout
