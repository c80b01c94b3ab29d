"""The sampler's kernels (csrc/sample.hip) on the host, a workgroup's wavefronts in orders that are chosen here: an access that lacks a
barrier gives a wrong token every time, and nothing of it has to run on a GPU to be seen."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import decode_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_27390_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"                             # (bf16 and fp16 as the kernels spell them)


def host_source(text):
    """Launches as calls; inline assembly, which is there for the choice of registers, as what it computes."""
    text, launches = re.subn(r"(\w+(?:<[\w, =]*>)?)<<<(.*?), (\w+), 0, stream>>>\((.*?)\);",
                             r"wavefronts::launch(\2, \3, [&] { \1(\4); });", text)
    assert launches >= 6 and "<<<" not in text
    text = text.replace('asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(x), "v"(y), "s"(c));', "d = fma(x, y, c);")
    text = text.replace('asm("" : "+v"(first));', "")
    assert "asm(" not in text
    return text


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    cc = shutil.which(CLANG)
    if cc is None:
        pytest.skip(f"no {CLANG}")
    tmp = tmp_path_factory.mktemp("sample")
    with open(os.path.join(CSRC, "sample.hip")) as f:
        (tmp / "sample.inc").write_text(host_source(f.read()))
    lib = str(tmp / "sample.so")
    res = subprocess.run([cc, "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-w", "-fsanitize=bounds", "-fsanitize-trap=bounds",
                          f'-DSAMPLE_SOURCE="{tmp / "sample.inc"}"', "-I", os.path.join(ROOT, "tests", "stub_wavefronts"), "-I", CSRC,
                          "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host_sample.cpp"), "-o", lib],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    lib = ctypes.CDLL(lib)
    lib.host_sample_workspace.restype = ctypes.c_size_t
    lib.host_sample.restype = ctypes.c_char_p
    return lib


TYPES = {"bf16": 0, "fp16": 1, "fp32": 2}
ORDERS = (0, 1, 2)                                               # the first wavefront first, the last one first, shuffled


def call(host, order, t, type, u, ids, kw):
    """One call: (tokens, logprobs)."""
    M, V = t.shape
    at = lambda x: None if x is None else ctypes.c_void_p(x.ctypes.data)   # noqa: E731
    got, lp = np.full(M, -7, np.int32), np.zeros(M, np.float32)
    ws = np.full(host.host_sample_workspace(M, V) + 256, 0xA5, np.uint8)
    error = host.host_sample(ctypes.c_uint(order), ctypes.c_void_p(t.data_ptr()), ctypes.c_longlong(V), TYPES[type], M, V, at(u),
                             at(kw.get("temperature")), at(kw.get("top_k")), at(kw.get("top_p")), at(kw.get("min_p")), at(ids), at(got),
                             at(lp), ctypes.c_void_p((ws.ctypes.data + 255) // 256 * 256))
    assert error is None, (order, error)
    return got, lp.astype(np.float64)


def args(z, u, kw):
    t, u, _, kw = inputs(z, u, "fp32", None, kw)
    return t, "fp32", u, None, kw


def inputs(z, u, type, ids, kw):
    import torch
    t = torch.from_numpy(np.asarray(z, dtype=np.float64)).to({"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[type])
    kw = {k: np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32) for k, v in kw.items()}
    return t, np.asarray(u, dtype=np.float32), None if ids is None else np.asarray(ids, dtype=np.int32), kw


def run(host, z, u, type="fp32", ids=None, orders=ORDERS, **kw):
    """Compares with the definition as the GPU's tests do, under every order; returns the tokens."""
    t, u, cols, kw = inputs(z, u, type, ids, kw)
    want, want_lp, margin = ref.sample(t.double().numpy(), u, ids=ids, **kw)
    sure = margin > 1e-11
    for order in orders:
        got, lp = call(host, order, t, type, u, cols, kw)
        assert np.array_equal(got[sure], want[sure]), (order, got, want)
        assert np.array_equal(np.isnan(lp[sure]), np.isnan(want_lp[sure])), order
        ok = sure & ~np.isnan(want_lp)
        assert (np.abs(lp - want_lp)[ok] <= 2.0 ** -23 * (1 + np.abs(want_lp[ok]))).all(), order
    return got


def test_lists_longer_than_twice_top_k(host):
    """What the slices hand on is counted, and cut to what can be among the k largest: two numbers that must not be one."""
    rng = np.random.default_rng(0)
    M, V = 4, 30000
    z = rng.standard_normal((M, V)) * 2
    run(host, z, rng.random(M), top_k=[2, 20, 50, 100], top_p=[0.9] * M, min_p=[0.01] * M)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("M,V", [(1, 1), (3, 1000), (2, 21000)])
def test_filters_in_every_order(host, type, M, V):
    rng = np.random.default_rng(M + V)
    z = rng.standard_normal((M, V)) * 2
    z[:, :: 7] = -np.inf
    for kw in ({}, dict(top_p=[0.8] * M), dict(top_k=[min(V, 300)] * M, top_p=[0.9] * M), dict(min_p=[0.02] * M),
               dict(temperature=[0.0] * M), dict(top_k=[5] * M)):
        run(host, z, rng.random(M), type, **kw)


def test_flat_rows_in_every_order(host):
    """More tokens at a border than lists hold: by digits of the keys."""
    rng = np.random.default_rng(3)
    z = np.zeros((2, 9000))
    run(host, z, rng.random(2), top_p=[0.5, 1.0], orders=(0, 1))
    run(host, z, rng.random(2), top_k=[200, 5000], orders=(0, 1))


def far_tokens(V):
    """Tokens that no row counts any more, but their slice does: the row's first 500 in its first half, and in the other half one
    at 2^-20 of them and the others at 2^-50 (or so: behind 2^-44 of the row's, not of the slice's)."""
    z = np.full(V, -np.inf)
    z[10:510] = -np.arange(500) * 1e-3
    z[V - 700] = -20 * np.log(2)
    z[V - 650:] = -50 * np.log(2) - np.arange(650) * 1e-3
    return z


def test_top_k_ends_behind_what_counts(host):
    """The bin that top-k cuts holds tokens of a slice that weigh nothing in the row, and no others."""
    M = 8
    z = np.tile(far_tokens(30000), (M, 1))
    u = (np.arange(M) + 0.5) / M
    for kw in ({}, dict(top_p=[0.97] * M), dict(min_p=[0.8] * M)):
        run(host, z, u, top_k=[600] * M, orders=(0,), **kw)


@pytest.mark.parametrize("top_k", [None, 600])
def test_last_bin_without_a_token(host, top_k):
    """A slice whose best token weighs 2^-43.99 of the row's first, and u of 1 and above, which ends with the last token that counts.  Tokens below
    2^-42 may be left out: the row's first token is as right as that one, and nothing else is."""
    z = np.full((1, 30000), -np.inf)
    z[0, 5], z[0, 29000] = 0.0, -43.99 * np.log(2)
    kw = {} if top_k is None else dict(top_k=[top_k])
    for u in (1.0, np.inf, np.nan):
        got, lp = call(host, 0, *args(z, [u], kw))
        assert got[0] in (5, 29000) and np.isfinite(lp[0])


@pytest.mark.parametrize("V", [40, 30000])
def test_min_p_above_one(host, V):
    """No token weighs more than 1: the first is kept, and those that tie with it are not."""
    z = np.zeros((3, V))
    z[:, 7:] = -np.arange(V - 7) - 1.0
    for kw in ({}, dict(top_k=[20] * 3), dict(top_k=[300] * 3), dict(top_p=[0.999] * 3)):
        assert run(host, z, [0.1, 0.5, 0.9], min_p=[1.5, 1.0000001, np.inf], orders=(0,), **kw).tolist() == [0, 0, 0]
        run(host, z, [0.1, 0.5, 0.9], min_p=[1.0, 1.0, 0.99], orders=(0,), **kw)


def test_slices_on_either_side_of_the_largest_quotient(host):
    """Logits of 2^22 temperatures: a row whose best lies just within what the bins take, and a slice whose best lies just past it."""
    V = 24000
    z = np.full((1, V), -np.inf)
    z[0, 3], z[0, V - 5] = -4.0 + 2.0 ** -21, -4.0
    for kw in ({}, dict(top_p=[0.9]), dict(top_k=[400]), dict(top_k=[4])):
        run(host, z, [0.8], temperature=[2.0 ** -20], orders=(0,), **kw)


def by_digits(host):
    """Whether the last call had a row that was ended digit by digit (about 0.8 ms of a workgroup for a row of 151,936)."""
    with open(os.path.join(CSRC, "sample.hip")) as f:
        text = f.read().split("\n")
    first = next(i for i, line in enumerate(text) if "u64 find_key(" in line)
    last = next(i for i, line in enumerate(text) if i > first and line == "}")
    lines = ctypes.POINTER(ctypes.c_int)()
    n = host.host_barriers(ctypes.byref(lines))
    assert n > 0
    return any(first < lines[i] - 1 < last for i in range(n))


def test_flat_rows_go_by_digits(host):
    run(host, np.zeros((1, 9000)), [0.5], top_p=[0.9], orders=(0,))
    assert by_digits(host)
    run(host, np.random.default_rng(5).standard_normal((1, 9000)), [0.5], top_p=[0.9], orders=(0,))
    assert not by_digits(host)


@pytest.mark.parametrize("allowed", [(0, 3000), (0, 900), (12000, 12400), (100, 28000)])
@pytest.mark.parametrize("mask", [-np.inf, -3.0e38, -1.0e4])
def test_top_k_of_a_range_of_columns(host, allowed, mask):
    """Only columns of a range are allowed, the others masked by whatever is low: wavefronts of a slice have all of them or none, and the
    masked ones are equal.  Neither is a reason to go through a row again and again."""
    rng = np.random.default_rng(6)
    M, V = 3, 30000
    z = np.full((M, V), mask)
    z[:, allowed[0]:allowed[1]] = rng.standard_normal((M, allowed[1] - allowed[0])) * 2
    run(host, z, rng.random(M), top_k=[3, 50, 250], top_p=[0.95] * M, orders=(0,))
    assert not by_digits(host)


def test_top_k_of_ranges_in_every_slice(host):
    """700 columns of each of 8 slices, few enough for each one's list and too many for the row's."""
    rng = np.random.default_rng(7)
    V = 8 * 20480
    z = np.full((1, V), -np.inf)
    for j in range(8):
        z[0, j * 20480 + 1000:j * 20480 + 1700] = rng.standard_normal(700)
    run(host, z, [0.7], top_k=[50], orders=(0,))
    assert not by_digits(host)


def test_top_k_over_slices_that_list_what_is_above_their_bound(host):
    """Each slice has fewer tokens above a common value than k, together they have more, or just as many, or fewer."""
    rng = np.random.default_rng(8)
    V = 30000
    for low in (-5.0, -1.0e4, -3.0e38):
        z = np.full((3, V), low)
        for m, each in enumerate((30, 25, 12)):
            for first in (0, 15000):
                at = first + rng.choice(15000, each, replace=False)
                z[m, at] = rng.standard_normal(each)
        run(host, z, rng.random(3), top_k=[50] * 3, orders=(0,))
        z[:, 100:200] = 3.0 + rng.standard_normal((3, 100))     # one slice has enough by itself
        run(host, z, rng.random(3), top_k=[50] * 3, orders=(0, 1))
        assert not by_digits(host)
