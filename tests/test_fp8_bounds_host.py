"""The figures of msa_fp8.h and the read-me, against the format's definition in 64 bits."""
import os
import re

import torch

from serve_ref import e4m3, exponent, pow2, quantise

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def text(*path):
    return re.sub(r"\s*\n \*\s*|\s+", " ", open(os.path.join(ROOT, *path), encoding="utf-8").read())


def test_bytes_of_a_token():
    """Eight heads of 128: K and V of a byte each, and a byte for each token and head of both."""
    want = 8 * 2 * (128 + 1)
    assert [int(x) for x in re.findall(r"(\d+) bytes a token", text("include", "msa_fp8.h"))] == [want]
    assert [int(x) for x in re.findall(r"(\d+) bytes a token", text("README.md"))] == [want]


def stated_bound():
    """(t, s): numbers from 2^-t of their row's largest on are off by 2^-4 of themselves at most, in rows whose
    largest is 2^-s or more."""
    (found,) = re.findall(r"at most 2\^-4, down to 2\^-(\d+) of its row's largest \(if that is 2\^-(\d+) or more\)",
                          text("include", "msa_fp8.h"))
    return int(found[0]), int(found[1])


def test_relative_error():
    t, s = stated_bound()
    # largest numbers at both ends of a power's range and between, from the smallest stated one on
    largest = torch.cat([torch.tensor([225.0, 224.5, 448.0, 300.0, 256.0], dtype=torch.float64) * pow2(torch.tensor(e))
                         for e in (-100, -30, -1, 0, 7, 100)] + [torch.tensor([2.0 ** -s, 1.01 * 2.0 ** -s], dtype=torch.float64)])
    part = pow2(torch.arange(-t, 0))[:, None] * torch.linspace(1.0, 2.0, 257, dtype=torch.float64)[None, :]
    x = largest[:, None] * torch.cat((torch.ones(1, dtype=torch.float64), part.flatten()))[None, :]
    y = quantise(x)[0]
    assert ((y - x).abs() <= x * 2.0 ** -4).all()
    # below: half the smallest step, 2^-10 of the power
    z = largest[:, None] * torch.cat((torch.ones(1, dtype=torch.float64), part.flatten() * 2.0 ** -t))[None, :]
    step = pow2(exponent(z))[:, None]
    assert ((quantise(z)[0] - z).abs() <= torch.maximum(z * 2.0 ** -4, step * 2.0 ** -10)).all()


def test_largest_numbers():
    """Every bf16 number below the stated limit is stored as a bf16 number; at the limit as 2^128, which is none."""
    (top,) = re.findall(r"finite and below (\d+) \* 2\^120", text("include", "msa_fp8.h"))
    limit = int(top) * 2.0 ** 120
    x = torch.arange(1 << 15, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x)].double()
    y = quantise(x[:, None])[0][:, 0]
    assert torch.equal(y.to(torch.bfloat16).double() == y, x < limit)
    assert torch.isfinite(y.float()).equal(x < limit) and bool((y[x >= limit] == 2.0 ** 128).all())
    assert float(e4m3(torch.tensor(247.99, dtype=torch.float64))) == 240.0
