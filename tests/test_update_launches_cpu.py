"""Launches of the update side's operators on the CPU, from one element to the largest sizes that the entry points take: the
host code against a recording stand-in for the HIP runtime (update_launches.hip).  A launch of 2^32 threads or more in a
dimension is refused by the runtime, after launches before it have already written."""
import ctypes
import os
import subprocess

import pytest

import paper_2608_11226_amd as R

PKG = os.path.dirname(os.path.abspath(R.__file__))
HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="no ROCm compiler here")


@pytest.fixture(scope="module")
def made(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    (d / "code").write_bytes(bytes(64))  # in the place of the device code, which is not compiled
    obj, lib = d / "launches.o", d / "launches.so"
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-fPIC", f"-I{PKG}/csrc",
                    f"-I{os.path.dirname(PKG)}/include", "-Xclang", "-fcuda-include-gpubinary", "-Xclang", str(d / "code"),
                    "-c", os.path.join(HERE, "update_launches.hip"), "-o", str(obj)], check=True, capture_output=True)
    subprocess.run(["g++", "-shared", str(obj), "-o", str(lib)], check=True, capture_output=True)
    so = ctypes.CDLL(str(lib))
    so.most_threads.restype = ctypes.c_uint64
    return so


MEMORY = 309 << 30  # more than the card has
SIZES = sorted({1, 3, 100} | {k + d for s in range(8, 31) for k in (1 << s, 3 << (s - 1)) for d in (-1, 0, 1)})
SIZES = [k for k in SIZES if k <= 1 << 30]


def test_embedding_gradients_of_every_size(made):
    seen = 0
    for vocab in SIZES:
        for dim in SIZES:
            # the smallest type; nothing larger than the memory is ever passed
            if 2 * vocab * dim > MEMORY:
                break
            for n in (1, 5, 6144, 6145, 32767, 32768, 1 << 20, 1 << 25, 1 << 28):
                if n * ((dim + 1023) // 1024) > 1 << 25 or 2 * n * dim > MEMORY:
                    break
                for acc in (0, 1):
                    assert made.embedding_backward(n, vocab, dim, 1, acc) == 0, (n, vocab, dim, acc, made.most_threads())
                    seen += 1
    assert seen > 10000


def test_other_calls_of_every_size(made):
    for rows in SIZES:
        for width in SIZES:
            if 2 * rows * width > MEMORY:
                break
            for bf16 in (0, 1):
                for top in (0, 1, 32):
                    if top <= width and not (top and width > 327680):
                        assert made.logprobs(rows, width, top, bf16) == 0, (rows, width, top, bf16)
                assert made.logprobs_backward(rows, width, bf16) == 0, (rows, width, bf16)
            if rows <= 1 << 28:
                assert made.embedding(rows, 1000, width) == 0, (rows, width)
            if rows * width < 1 << 31:
                assert made.policy_loss(rows, width, 1) == 0, (rows, width)
