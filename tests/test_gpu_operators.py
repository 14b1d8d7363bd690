"""The cases of perf/operators.py at their own sizes, and some drawn from the same ranges: the library's results and the file's own 64-bit forms
against tests/plain64.py with its bounds."""
import importlib.util
import os
import random

import pytest
import torch

import plain64

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_spec = importlib.util.spec_from_file_location("operators_cases", os.path.join(ROOT, "perf", "operators.py"))
operators = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(operators)

CASES = {c["name"]: c for c in operators.listed()}
CASES.update(("drawn_%d" % i, operators.draw(random.Random(i))) for i in range(12))


def _same(exact, want):
    """Two 64-bit forms of one thing: angles of up to 2^18 radians are off by 2^-34, sums of 10^5 terms by less."""
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(exact), inf)
    assert float((exact - want)[~inf].abs().max()) <= 1e-9 * max(1.0, float(want[~inf].abs().max()))


@pytest.mark.parametrize("name", CASES)
def test_case(lazyev_lib, monkeypatch, name):
    monkeypatch.setattr(operators, "own", True)
    case, seed = CASES[name], 77
    state = operators.prepare(case, seed)
    before = {x: state[x].clone() for x in ("k_pages", "v_pages") if x in state}
    got, exact = operators.run(state), operators.exact(case, seed)
    S, T = case["seqs"], case["tokens"]
    if case["kind"] == "rotate":
        for x in ("q", "k"):
            want, bound = plain64.turn(state[x], state["positions"], state[x + "_weight"], operators.EPS, state["inv_freq"], case["layout"])
            plain64.check_out(got[x], want, bound)
            _same(exact[x], want)
    elif case["kind"] == "append":
        at = case["start"] + torch.arange(T, device="cuda")
        want, bound = plain64.turn(state["k"], at.expand(S, T), state["k_weight"], operators.EPS, state["inv_freq"], case["layout"])
        pages, places = state["table"].long()[:, at // case["page"]], (at % case["page"]).expand(S, T)
        plain64.check_out(got["k_pages"][pages, :, places], want, bound)
        _same(exact["k_pages"][pages, :, places], want)
        before["v_pages"][pages, :, places] = state["v"]
        assert torch.equal(got["v_pages"], before["v_pages"]) and torch.equal(exact["v_pages"], before["v_pages"].double())
        got["k_pages"][pages, :, places] = before["k_pages"][pages, :, places]
        assert torch.equal(got["k_pages"], before["k_pages"])
    else:
        length = case["length"]
        for s in range(S):
            k, v = (state[x][state["table"][s].long()].transpose(1, 2).flatten(0, 1)[:length] for x in ("k_pages", "v_pages"))
            vis = torch.full((T,), length, device="cuda") if state["visible"] is None else state["visible"][s].long()
            joined = None if state["joined"] is None else tuple(x[s] for x in state["joined"])
            want, lse, bound, bound_lse = plain64.attend(state["q"][s], k, v, vis, case["dim"] ** -0.5, joined)
            plain64.check_out(got["out"][s], want, bound)
            plain64.check_lse(got["lse"][s], lse, bound_lse)
            _same(exact["out"][s], want)
            _same(exact["lse"][s], lse)
