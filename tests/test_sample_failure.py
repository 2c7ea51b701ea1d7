"""What the sampling call does when one of its searches finds no token (CPU, by
reading the source; no input is known that brings it there).  The error word must
not say that a wait ran out, and the row must not keep an old token."""
import os
import re

from test_boundary_cpu import ROOT, ppas  # noqa: F401


def _read(*path):
    with open(os.path.join(ROOT, *path), encoding="utf-8") as f:
        return f.read()


def test_device_error_codes_of_header_and_binding(ppas):  # noqa: F811
    codes = dict(re.findall(r"#define (PPAS_DEVERR_[A-Z_]+) (\d+)", _read("include", "ppas.h")))
    assert codes["PPAS_DEVERR_SEARCH"] == "3" and len(set(codes.values())) == len(codes)
    for name, code in codes.items():
        assert getattr(ppas, name) == int(code)


def test_a_failed_search_has_its_own_code_and_leaves_no_old_token():
    text = re.sub(r"//[^\n]*", "", _read("paper_2608_15171_gb300", "csrc", "sample.cu"))
    assert "PPAS_DEVERR_TIMEOUT" not in text
    # one place reports, and writes what a row without a token has
    assert text.count("report_error(") == 1
    at = text.index("report_error(p.err, PPAS_DEVERR_SEARCH)")
    body = text[text.rindex("{", 0, at):text.index("};", at)]
    assert "p.tokens[r] = -1;" in body and "p.logprobs[r] = -INFINITY;" in body
