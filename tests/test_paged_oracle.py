"""Pins of the paged cache's float64 oracle that need no GPU: the page format against the header's formulas, the rotation against
complex numbers, quantisation errors against their bound, selection and attention against torch."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O


@pytest.mark.parametrize("P,D", [(32, 64), (64, 128), (128, 64)])
@pytest.mark.parametrize("keys", [True, False])
def test_every_code_and_scale_has_a_place_of_its_own(P, D, keys):
    at = np.array([[O.places(keys, r, d, D) for d in range(D)] for r in range(P)])
    codes = at[..., 0] * 8 + at[..., 1]
    assert sorted(codes.ravel()) == list(range(P * D))
    scales = np.concatenate([at[..., 2].reshape(P, D // 32, 32), at[..., 3].reshape(P, D // 32, 32)])
    assert (scales == scales[..., :1]).all() and sorted(scales[..., 0].ravel()) == list(range(2 * P * (D // 32)))


@pytest.mark.parametrize("D", [64, 128])
def test_places_follow_the_headers_formulas(D):
    for r, g, s, e in ((0, 0, 0, 0), (37, 1, 2, 5), (63, D // 32 - 1, 3, 7), (50, 0, 1, 6)):
        gp = [0, 2, 1, 3][g] if D == 128 else g
        assert O.places(True, r, 32 * g + 8 * s + e, D) == (r * D // 8 + s * D // 32 + gp, e // 2 + 4 * (e % 2), 2 * (r * D // 32 + gp), 2 * (r * D // 32 + gp) + 1)
    for t, q, i, far, j, w, m in ((0, 0, 0, 0, 0, 0, 0), (1, 2, 3, 1, D // 64 - 1, 3, 15), (2, 3, 1, 0, 0, 2, 7)):
        r, d, e = 32 * t + 16 * far + 4 * q + i, 64 * j + 16 * w + m, 2 * i + far
        at = ((4 * t + q) * D // 32 + d // 32) * 16 + e
        assert O.places(False, r, d, D) == ((4 * t + q) * D + 64 * j + 4 * m + w, e // 2 + 4 * (e % 2), at, at + 8)


@pytest.mark.parametrize("fmt,dtype", [("rows", "f32"), ("rows", "bf16"), ("4bit", "bf16")])
@pytest.mark.parametrize("keys", [True, False])
def test_written_rows_read_back_and_leave_the_others(fmt, dtype, keys):
    P, D = 32, 64
    rng = np.random.default_rng(3)
    page = rng.integers(0, 256, O.page_bytes(fmt, dtype, P, D), dtype=np.uint8)
    before = page.copy()
    rows = O.as_dtype(rng.standard_normal((P, D)), dtype)
    for r in (0, 7, 19, 31):
        O.write_row(page, fmt, dtype, keys, P, r, rows[r])
    got, old = O.read_rows(page, fmt, dtype, keys, P, D), O.read_rows(before, fmt, dtype, keys, P, D)
    for r in range(P):
        if r not in (0, 7, 19, 31):
            assert np.array_equal(got[r], old[r], equal_nan=True)
        elif fmt == "rows":
            assert np.array_equal(got[r], rows[r])
        else:
            code, step, base = O.quantise(rows[r])
            assert np.array_equal(got[r], O.element(code, np.repeat(step, 32), np.repeat(base, 32)))


def test_quantisation_error_is_half_a_code():
    """|x - element| <= S / 32 for codes inside 0 ... 15.  The ends add what rounding to fp16 moves them: base and step together by
    half a unit of |B| + S, 2^-11 of it; fp16 below 2^-14 has absolute steps of 2^-24."""
    rng = np.random.default_rng(4)
    for scale, offset in ((1, 0), (30, 0), (0.05, 1), (1, 40), (1e-3, 0), (2000, -3000)):
        x = O.as_dtype(rng.standard_normal(4096) * scale + offset, "bf16")
        code, step, base = O.quantise(x)
        s, b = np.repeat(step.astype(float), 32), np.repeat(base.astype(float), 32)
        err = np.abs(x - (b + s * (1 + code / 16)))
        assert (err <= s / 32 + 2.0 ** -10 * (np.abs(b) + s) + 2.0 ** -23).all()
    x = np.array([3.0] * 32 + [1e6, -1e6] * 16)
    code, step, base = O.quantise(x)
    assert step[0] == 0 and code[:32].max() == 0 and base[0] == 3 and np.isfinite(step).all() and np.isfinite(base).all()


def test_rotation_is_a_complex_product():
    rng = np.random.default_rng(5)
    half = 32
    angle = rng.random((50, half)) * 6
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    x = rng.standard_normal(2 * half).astype(np.float32).astype(np.float64)
    for sections, pos in ((None, [7]), ((5, 0, 27), [3, 9, 49]), ((0, 32, 0), [1, 2, 3])):
        axis = [0] * half if sections is None else [0] * sections[0] + [1] * sections[1] + [2] * sections[2]
        z = [(x[i] + 1j * x[i + half]) * (float(cos[pos[axis[i]], i]) + 1j * float(sin[pos[axis[i]], i])) for i in range(half)]
        want = np.array([v.real for v in z] + [v.imag for v in z])
        got = O.rotate(x, cos, sin, pos, sections, "f32")
        assert np.abs(got - want).max() <= 2.0 ** -23 * np.abs(want).max()
    assert np.array_equal(O.rotate(x, cos, sin, [99], None, "f32"), O.rotate(x, cos, sin, [49], None, "f32"))     # clamped


def test_selection_and_attention_against_torch():
    rng = np.random.default_rng(6)
    s = rng.integers(0, 6, 40).astype(np.float32)                      # many equal scores
    for keep, first, last in ((8, 1, 1), (12, 0, 3), (39, 2, 0), (40, 1, 1), (5, 5, 0)):
        t = torch.from_numpy(s.copy())
        t[:first] = np.inf
        t[len(s) - last:] = np.inf
        order = torch.sort(t, descending=True, stable=True).indices[:keep]
        assert O.select(s, keep, first, last) == sorted(order.tolist())
    q, k, v = rng.standard_normal((3, 16)), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    want = torch.softmax(torch.from_numpy(0.3 * (q @ k.T)), -1) @ torch.from_numpy(v)
    assert np.abs(O.attention(q, k, v, 0.3) - want.numpy()).max() < 1e-12
    assert (O.attention(q, k[:0], v[:0], 1.0) == 0).all()
    gone = k.copy()
    gone[:, 0], q[:, 0] = -np.inf, 1.0
    assert (O.attention(q, gone, v, 1.0) == 0).all()


def test_page_scores_bound_every_key_between_the_bounds():
    rng = np.random.default_rng(7)
    Hkv, G, D, P = 2, 3, 8, 32
    table, lengths = np.array([[[1, 0, -1], [2, 2, 0]]]), np.array([[70, 40]])
    lo = rng.standard_normal((3, 1, D))
    bounds = np.concatenate([lo, lo + rng.random((3, 1, D))], 1)
    Q = rng.standard_normal((1, Hkv * G, D))
    got = O.page_scores(Q, bounds, table, lengths, P, 0, 0)
    assert len(got) == 3 and got[2] == -np.inf and len(O.page_scores(Q, bounds, table, lengths, P, 0, 1)) == 2
    for page, score in ((1, got[0]), (0, got[1])):
        corners = sum(max(q[d] * bounds[page, 0, d], q[d] * bounds[page, 1, d]) for q in Q[0, :G] for d in range(D))
        assert abs(score - corners) < 1e-5
