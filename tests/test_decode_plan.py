"""How the attention over a cache divides its calls, and the workspace that it asks for:
on the CPU over drawn sizes, plainly and under AddressSanitizer and
UndefinedBehaviorSanitizer; on the GPU the calls of few rows whose tables name more keys
than the workspace holds logits for."""
import os
import subprocess

import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, host, say  # noqa: F401
from test_sanitizers import SAN

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.mark.parametrize("flags", (["-O2"], SAN), ids=("plain", "sanitizers"))
def test_plans(tmp_path, flags):
    out = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", *flags, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2111_13824_amd", "csrc"),
                    os.path.join(HERE, "decode_plan_main.cpp"), "-o", out], check=True)
    env = {k: v for k, v in os.environ.items() if k != "LD_PRELOAD"}
    r = subprocess.run([out], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-2000:]
    *ways, largest = map(int, r.stdout.split())
    assert all(n > 1000 for n in ways) and largest > 1 << 29


# (B, Hq, Hkv, L, d, page, lengths, what a table names, scale, depth): one launch and parts
WIDE = [(9, 16, 2, 2, 64, 64, [300, 1, 0, 77, 2000, 64, 5, 1300, 63], 1 << 20, 2.0 ** -10, 20),
        (18, 15, 1, 1, 128, 32, [64, 700, 65, 0] * 4 + [1, 2], 1 << 20, 2.0 ** -10, 20),
        (12, 64, 8, 1, 16, 16, [33 * i for i in range(12)], 1 << 19, 0.1, 26),
        (40, 16, 16, 1, 32, 16, [5 + 9 * i for i in range(40)], 1 << 19, 2.0 ** -10, 20),
        (36, 16, 16, 2, 48, 128, [130] * 36, 1 << 19, 2e-4, 14),
        (33, 8, 4, 1, 64, 1024, [40 * i for i in range(33)], 1 << 20, 2.0 ** -10, 20)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "x".join(map(str, c[:6])))
def test_tables_of_more_keys_than_logits_are_kept_for(fq, case):  # noqa: F811
    B, Hq, Hkv, L, d, page, length, most, s, n = case
    rows = L * Hq // Hkv
    need = fq.lis_attention_paged_workspace_bytes(B, Hq, Hkv, L, d, most)
    assert rows <= 16 and 4 * B * Hkv * rows * most > 1 << 30 > 1 << 20 > need
    c, q, length, n_new, _, _ = R.attend_case((B, Hq, Hkv, L, d, page, length, [L] * B, {}))
    ref, grown = R.attend(c, q, length, n_new, s, zp_q=3, zp_v=-5, n=n)
    table = np.full((B, most // page), -1, np.int32)
    table[:, :c["table"].shape[1]] = c["table"]
    w = dev(c["weight"])
    say("wide tables", case[:6], need)
    for weight in (None, w):
        out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(table), dev(length), s, zp_q=3, zp_v=-5,
                                     exp_n=n, weight=weight)
        assert np.array_equal(host(out), ref)
    assert np.array_equal(host(w), c["weight"] + grown)
