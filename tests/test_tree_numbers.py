"""Host parts of a speculative step: the numbers that its operators are held in, and the store of TMA maps."""
import decimal
import os
import shutil
import subprocess
from decimal import Decimal as D

import numpy as np
import pytest

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
@pytest.mark.parametrize("name", ["tree_fixed", "map_store"])
def test_host_parts(name, tmp_path):
    """tests/c: probabilities in fixed point, and the store of TMA maps."""
    exe = tmp_path / name
    cc = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error",
                         "-I", os.path.join(ROOT, "paper_2607_16213_gb300", "csrc"),
                         os.path.join(ROOT, "tests", "c", name + ".cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert cc.returncode == 0, cc.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout.strip() == "done", (run.returncode, run.stdout + run.stderr)


TWO_PI = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")


def exact_turns(rot, theta, scaling=None, factor=1.0, original=0, low=1.0, high=32.0):
    """Each pair's turns a position, from the formula in 80 digits."""
    with decimal.localcontext() as c:
        c.prec = 80
        theta, factor, low, high = D(theta), D(factor), D(low), D(high)
        out = []
        for f in range(rot // 2):
            t = (-D(2 * f) / rot * theta.ln()).exp() / TWO_PI
            if scaling == "linear":
                t = t / factor
            elif scaling is not None:
                if scaling == "wavelength":
                    keep = (original * t - low) / (high - low)
                else:
                    at = lambda n: rot * (D(original) / (TWO_PI * n)).ln() / (2 * theta.ln())  # noqa: E731
                    i0 = max(D(0), at(high).to_integral_value(decimal.ROUND_FLOOR))
                    i1 = min(D(rot - 1), at(low).to_integral_value(decimal.ROUND_CEILING))
                    keep = 1 - (f - i0) / max(i1 - i0, D(0.001))
                keep = min(D(1), max(D(0), keep))
                t = keep * t + (1 - keep) * t / factor
            out.append(t)
        return out


PLANS = [dict(rot=128, theta=1e4), dict(rot=128, theta=5e5), dict(rot=64, theta=1e6), dict(rot=2, theta=1e4), dict(rot=6, theta=1.0),
         dict(rot=18, theta=0.5), dict(rot=34, theta=1e-6), dict(rot=16, theta=1e300), dict(rot=2, theta=5e-324), dict(rot=30, theta=1.0 + 2.0 ** -40),
         dict(rot=128, theta=1e4, scaling="linear", factor=3.7), dict(rot=128, theta=5e5, scaling="linear", factor=1e-3),
         dict(rot=128, theta=5e5, scaling="wavelength", factor=8.0, original=8192, low=1.0, high=4.0),
         dict(rot=120, theta=1e4, scaling="wavelength", factor=1.3, original=100, low=0.1, high=3.3),
         dict(rot=64, theta=1e4, scaling="ramp", factor=16.0, original=4096, low=1.0, high=32.0),
         dict(rot=128, theta=1.5e5, scaling="ramp", factor=40.0, original=4096, low=1.0, high=32.0),
         dict(rot=32, theta=10.0, scaling="ramp", factor=2.0, original=64, low=1.0, high=1e6)]


@pytest.fixture
def lib():
    from paper_2607_16213_gb300 import build as b
    b.build()
    return S.library()


@pytest.mark.parametrize("kw", PLANS, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_rotary_plan_is_right_to_its_last_bit(lib, kw):
    """turns: rounded to units of 2^-64, so half of one off, and a hundredth for the 2^-90 of the arithmetic before that (turns below 2^19)."""
    plan = api.rotary_plan(kw["rot"], kw["theta"], **{k: v for k, v in kw.items() if k not in ("rot", "theta")})
    with decimal.localcontext() as c:
        c.prec = 80
        for f, t in enumerate(exact_turns(**kw)):
            off = abs(D(plan.turns[f]) - t * D(2) ** 64) % D(2) ** 64
            assert min(off, D(2) ** 64 - off) <= D("0.51"), (f, float(off))


@pytest.mark.parametrize("kw", PLANS, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_angles_of_far_positions(lib, kw):
    """What the kernel takes of a plan, the upper half of position times turns, is right to 2^-31 turns: 2^-34 for the rounded
    turns at 2^31 positions, 2^-32 cut off."""
    plan = api.rotary_plan(kw["rot"], kw["theta"], **{k: v for k, v in kw.items() if k not in ("rot", "theta")})
    rng = np.random.default_rng(7)
    with decimal.localcontext() as c:
        c.prec = 80
        for f, t in enumerate(exact_turns(**kw)):
            for p in [2 ** 31 - 1, -2 ** 31] + [int(x) for x in rng.integers(-2 ** 31, 2 ** 31, 6)]:
                turn = D(((p * plan.turns[f]) % 2 ** 64) >> 32) / D(2) ** 32
                off = abs(turn - p * t) % 1
                assert min(off, 1 - off) <= D(2) ** -31, (f, p)
