"""The pins of the oracle's operators for activations without a calibrated grid catch plausible mistakes
(no GPU): each case plants one in a copy of the C oracle, which must then fail
a pin of PIN_FILES in a child process, as in test_oracle_mutants.py."""

import concurrent.futures as cf
import os

import pytest

from tests import test_oracle_mutants as harness

PIN_FILES = ["test_oracle_operators.py", "test_oracle_operators_bits.py"]

# (name, [(text in the oracle, planted replacement), ...])
MUTANTS = [
    ("quantize: alpha past the type's grid", [("    if (alpha > lim) alpha = lim;\n", "")]),
    ("quantize: ties rounded down", [
        ("floor_div(254 * (int64_t)x[r * d + k] + alpha, 2 * alpha)",
         "floor_div(254 * (int64_t)x[r * d + k] + alpha - 1, 2 * alpha)")]),
    ("quantize: scale of half the size", [
        ("alpha * ((int64_t)1 << (32 - bits))", "alpha * ((int64_t)1 << (31 - bits))")]),
    ("quantize: largest value without its sign", [
        ("const int64_t v = x[r * d + k], av = v < 0 ? -v : v;", "const int64_t v = x[r * d + k], av = v;")]),
    ("linear: no residual term", [("      if (z) v += (__int128)m_z", "      if (0) v += (__int128)m_z")]),
    ("linear: residual term in other units", [("m_z * 65536 * z[", "m_z * 32768 * z[")]),
    ("linear: no bias", [("t * mult[c] + (bias ? bias[c] : 0) + two_n / 2", "t * mult[c] + two_n / 2")]),
    ("linear: output rounded down", [("(bias ? bias[c] : 0) + two_n / 2", "(bias ? bias[c] : 0)")]),
    ("linear: token product toward zero", [
        ("floor_div128((__int128)acc * ((int64_t)1 << p) * s[r], (__int128)1 << 32)",
         "(__int128)acc * ((int64_t)1 << p) * s[r] / ((__int128)1 << 32)")]),
    ("linear: one bit less of the product", [("  int32_t p = 16;", "  int32_t p = 15;")]),
    ("linear: scale of another token", [("((int64_t)1 << p) * s[r]", "((int64_t)1 << p) * s[0]")]),
    ("linear: weights transposed", [
        ("w[(int64_t)c * d_in + k];\n      const __int128 t", "w[(int64_t)k * d_out + c];\n      const __int128 t")]),
    ("linear: multiplier of the first channel", [("t * mult[c] +", "t * mult[0] +")]),
    ("group norm: padded frames in the statistics", [
        ("for (int32_t t = 0; t < L; ++t)\n        for (int32_t c = g * cg;",
         "for (int32_t t = 0; t < T; ++t)\n        for (int32_t c = g * cg;"),
        ("const __int128 n = (__int128)L * cg;", "const __int128 n = (__int128)T * cg;")]),
    ("group norm: padded frames written", [
        ("for (int32_t t = 0; t < L; ++t) {\n          const int64_t at",
         "for (int32_t t = 0; t < T; ++t) {\n          const int64_t at")]),
    ("group norm: count of the padded frames", [
        ("const __int128 n = (__int128)L * cg;", "const __int128 n = (__int128)T * cg;")]),
    ("group norm: remainder of the mean left in the deviations", [(" - floor_div128(r * r, n);", ";")]),
    ("group norm: deviations rounded down", [("- floor_div128(r * r, n);", "+ floor_div128(-r * r, n);")]),
    ("group norm: mean toward zero", [("floor_div128(S * 131072 + n, 2 * n)", "(S * 131072 + n) / (2 * n)")]),
    ("group norm: mean rounded down", [("floor_div128(S * 131072 + n, 2 * n)", "floor_div128(S * 131072, 2 * n)")]),
    ("group norm: no mean", [("D->gn_bias[c] - floor_div128(mu * A, 65536)", "D->gn_bias[c]")]),
    ("group norm: no bias", [("D->gn_bias[c] - floor_div128(mu * A, 65536)", "-floor_div128(mu * A, 65536)")]),
    ("group norm: eps of one", [("(V + D->eps) * 65536", "(V + 1) * 65536")]),
    ("group norm: root one too large", [
        ("ipk_oracle_isqrt((int64_t)((V + D->eps) * 65536));",
         "ipk_oracle_isqrt((int64_t)((V + D->eps) * 65536)) + 1;")]),
    ("group norm: multiplier of half the size", [
        ("(__int128)1 << (40 - D->in_bits)", "(__int128)1 << (41 - D->in_bits)")]),
    ("group norm: output rounded down", [("z[at] * A + C + ((__int128)1 << (D->gn_shift - 1))", "z[at] * A + C")]),
    ("group norm: Swish of values past int16", [
        ("const int64_t h16 = clamp_bits(h, 16);", "const int64_t h16 = (int64_t)h;")]),
    ("group norm: gamma of the group's first channel", [("D->gn_mult[c] * R", "D->gn_mult[g * cg] * R")]),
    ("operators: grids down to their lowest value", [
        ("return v < -lim ? -lim : (v > lim", "return v < -lim - 1 ? -lim - 1 : (v > lim")]),
]


def test_every_planted_mistake_fails_a_pin(tmp_path, monkeypatch):
    monkeypatch.setattr(harness, "PIN_FILES", PIN_FILES)
    with cf.ThreadPoolExecutor(max(2, min(6, (os.cpu_count() or 4) - 2))) as pool:
        results = list(pool.map(lambda m: (m[0],) + harness._failed_pins(m[0], m[1], str(tmp_path)),
                                MUTANTS + [("unchanged", [])]))
    missed = []
    for name, rc, failed in results:
        print(f"[mutant] {name}: {rc=} caught by {failed}")
        if name == "unchanged":
            assert rc == 0 and not failed, failed
        elif rc == 0 or not failed:
            missed.append(name)
    assert not missed, f"planted mistakes no pin catches: {missed}"


@pytest.mark.parametrize("name", [m[0] for m in MUTANTS])
def test_each_planted_text_is_in_the_oracle(name):
    src = open(harness.SRC).read()
    for old, _ in dict(MUTANTS)[name]:
        assert src.count(old) == 1
