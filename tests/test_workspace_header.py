"""The words of the workspace header: no operator's overlap another's."""

import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_16798_gb300", "csrc")


def _compiles(tmp_path, slots=None, offset=None):
    """Whether the summary's assertion holds, as it is or with another number of slots or place of the first."""
    src = open(os.path.join(CSRC, "rl_stats.cu")).read()
    host = open(os.path.join(CSRC, "rl_host.h")).read()
    n, check = (re.search(p, src, re.S).group(0) for p in (r"constexpr int kSumSlots = \d+;", r"static_assert\([^;]*kSumSlots[^;]*;"))
    if slots:
        n = re.sub(r"\d+", str(slots), n)
    if offset:
        host, count = re.subn(r"(kWsSummaryOffset = )\d+", rf"\g<1>{offset}", host)
        assert count == 1
    (tmp_path / "rl_host.h").write_text(host)
    f = tmp_path / "check.cpp"
    f.write_text(f'#include "rl_host.h"\nnamespace rl {{\n{n}\n{check}\n}}\n')
    r = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I",
                        "/usr/local/cuda/include", str(f)], capture_output=True, text=True)
    return r.returncode == 0, r.stderr


def test_summary_slots_are_held_off_the_next_words(tmp_path):
    """One more cluster's totals, or the same ones eight bytes on, would run into the words behind them: the build says so."""
    ok, err = _compiles(tmp_path)
    assert ok, err
    for change in (dict(slots=6), dict(offset=40)):
        ok, err = _compiles(tmp_path, **change)
        assert not ok and "static assertion failed" in err


@pytest.mark.gpu
def test_operators_in_turn_on_one_workspace():
    import torch

    from paper_2608_16798_gb300 import build

    build.build()
    import paper_2608_16798_gb300.rl_loss as R
    import verify_cases as VC

    rows = 50000  # as many clusters as have slots
    g = torch.Generator(device="cuda").manual_seed(1)
    stats = torch.rand(rows * 5, generator=g, device="cuda")
    mask = torch.ones(rows, dtype=torch.uint8, device="cuda")
    traj, coef = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    c = VC.make([2, 3, 1], 700, "f32", True, seed=1)
    ref = VC.expected(c)
    dev = [torch.from_numpy(np.ascontiguousarray(c[k])).cuda() for k in ("ids", "offsets", "u", "s")]
    z, zd = (torch.from_numpy(c[k]).float().cuda() for k in ("target", "draft"))
    grad = torch.randn(300, 400, generator=g, device="cuda")
    ws = R.new_muon_workspace(1, 300, 400)
    assert ws.numel() >= R.rl_workspace_size(rows, 700)
    first = None
    for _ in range(3):
        total = R.rl_token_stats_summary(stats, mask, traj, coef, ws)
        out, acc, _ = R.rl_verify_drafts(z, *dev, 3, R.make_verify_params(), ws, draft_logits=zd)
        update = R.rl_muon_update(grad, R.make_muon_params(momentum=0.0), ws)
        assert R.rl_query_status(ws)[1] == 0
        assert np.array_equal(out.cpu().numpy(), ref[0]) and np.array_equal(acc.cpu().numpy(), ref[1])
        now = (total.cpu(), update.cpu())
        first = now if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(first, now)) and total[0].item() == rows
