"""The normal distribution of the activations, from its coefficients in the source: its tail polynomial in 64 and in 32 bits."""
import os
import re

import numpy as np
from scipy.special import erfc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2407_19644_amd", "csrc", "ubp_device.h")
f32 = np.float32


def source():
    with open(HEADER) as f:
        text = f.read()
    body = text[text.index("float normal_cdf(float v, float &density)"):]
    body = body[:body.index("\n}\n")]
    first = float(re.search(r"float q = (\S+)f;", body).group(1))
    c = [first] + [float(v) for v in re.findall(r"q = fmaf\(q, t, (\S+?)f\)", body)]
    assert len(c) == 9 and all(float(f32(v)) == v for v in c)
    comment = text[:text.index("float normal_cdf(float v, float &density)")].rsplit("\n}\n", 1)[1]
    return c, " ".join(comment.replace("//", " ").split())


def fma(a, b, c):
    """A product and a sum rounded once: in 64 bits the product of two fp32 values is exact, and the sum's own rounding there is far
    below fp32's."""
    return (a.astype(np.float64) * b.astype(np.float64) + c).astype(f32)


def tail64(c, z):
    t = 1.0 / (1.0 + float(f32(0.3)) * z)
    q = np.zeros_like(z)
    for v in c:
        q = q * t + v
    return q * np.exp(-0.5 * z * z)


def tail32(c, z):
    z = z.astype(f32)
    t = (1.0 / fma(np.full_like(z, f32(0.3)), z, 1.0).astype(np.float64)).astype(f32)
    density = np.exp2((z * z * f32(-0.72134752044)).astype(np.float64)).astype(f32)
    q = np.full_like(z, f32(c[0]))
    for v in c[1:]:
        q = fma(q, t, v)
    return (q * density).astype(np.float64)


def test_the_stated_errors_are_the_coefficients():
    c, comment = source()
    z = np.linspace(0.0, 14.5, 1450001)
    want = 0.5 * erfc(z / np.sqrt(2.0))
    worst = np.abs(tail64(c, z) / want - 1).max()
    z5 = z[z <= 5].astype(f32).astype(np.float64)
    z10 = z[z <= 10].astype(f32).astype(np.float64)
    w5, w10 = 0.5 * erfc(z5 / np.sqrt(2.0)), 0.5 * erfc(z10 / np.sqrt(2.0))
    e5, e10 = (np.abs(tail32(c, a) / b - 1).max() for a, b in ((z5, w5), (z10, w10)))
    q = tail32(c, z5).astype(f32)
    absolute = max(np.abs(q - w5).max(), np.abs((f32(1) - q).astype(np.float64) - 0.5 * erfc(-z5 / np.sqrt(2.0))).max())
    print(worst, absolute, e5, e10)
    stated = [float(v) for v in re.findall(r"\d(?:\.\d+)?e-\d", comment)]
    assert len(stated) == 4, comment                                      # polynomial; Phi in fp32; its tail to z = 5, to z = 10
    for got, said in zip((worst, absolute, e5, e10), stated):
        assert 0.8 * said <= got <= said, (got, said)
