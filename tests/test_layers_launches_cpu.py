"""Launches of the layers' operators on the CPU, from one token to the largest sizes that the entry points take: the host code
against a recording stand-in for the HIP runtime (layers_launches.hip)."""
import ctypes
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

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
    sources = [os.path.join(PKG, "csrc", f + ".hip") for f in ("packed_attention", "packed_attention_backward", "rms_norm", "adamw")]
    sources.append(os.path.join(HERE, "layers_launches.hip"))

    def build(src):
        obj = d / (os.path.basename(src) + ".o")
        subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-fPIC", f"-I{PKG}/csrc",
                        f"-I{os.path.dirname(PKG)}/include", "-Xclang", "-fcuda-include-gpubinary", "-Xclang", str(d / "code"),
                        "-c", src, "-o", str(obj)], check=True, capture_output=True)
        return str(obj)

    with ThreadPoolExecutor(5) as ex:
        objs = list(ex.map(build, sources))
    lib = d / "launches.so"
    subprocess.run(["g++", "-shared", *objs, "-o", str(lib)], check=True, capture_output=True)
    so = ctypes.CDLL(str(lib))
    so.adamw.argtypes = [ctypes.c_int, ctypes.c_int64]
    return so


TOKENS = [1, 2, 31, 127, 128, 129, 1000, 4096, 8191, 65536, (1 << 20) + 1, 1 << 22, 1 << 26]


def test_attention_of_every_size(made):
    seen = 0
    for heads, kv in ((1, 1), (4, 4), (28, 4), (64, 8), (64, 1), (128, 2)):
        for hd in (32, 64, 128):
            for n_q in TOKENS:
                for n_k in (n_q, 1, 100000, (1 << 26) // heads):
                    for seqs in (1, 7, 300, 100000, 1 << 20):
                        s = R.AttentionShape(dtype=1, n_heads=heads, n_kv_heads=kv, head_dim=hd, n_seqs=seqs, n_q=n_q, n_k=n_k,
                                             causal=seqs & 1, scale=1.0)
                        try:
                            room = R.rollout_attention_workspace(s), R.rollout_attention_backward_workspace(s)
                        except R.RolloutError:
                            continue
                        assert 0 < room[0] <= 256 << 20 and room[1] <= (256 << 20) + 8 * n_q * heads + 16
                        for bf16 in (0, 1):
                            args = (bf16, heads, kv, hd, seqs, n_q, n_k, seqs & 1)
                            assert made.attention(*args) == 0 and 1 <= made.launches() <= 2, args
                            assert made.attention_backward(*args) == 0 and 2 <= made.launches() <= 4, args
                            seen += 1
    assert seen > 5000


def test_norms_of_every_size(made):
    seen = 0
    for rows in [1, 3, 4, 5, 1023, 1025, 4097, 1 << 20, (1 << 22) - 1, 1 << 22, 1 << 23, (1 << 26) - 1, 1 << 26]:
        for dim in (1, 8, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32768):
            try:
                R.rollout_rms_norm_backward_workspace(rows, dim)
            except R.RolloutError as e:
                assert e.code == R.EUNSUPPORTED and rows >= 1 << 22
                continue
            for x, delta, y in ((0, -1, 0), (0, 1, 1), (1, 0, 3), (1, 1, 3)):
                assert made.norm(rows, dim, x, delta, y) == 0 and made.launches() == 1, (rows, dim)
            for dgain in (0, 1):
                assert made.norm_backward(rows, dim, dgain) == 0 and made.launches() == 1 + dgain, (rows, dim)
            seen += 1
    assert seen > 120


def test_adamw_of_every_size(made):
    for chunks in (1, 1000, (1 << 24) - 8):
        assert made.adamw(1, chunks) == 0 and made.launches() == 1


def test_tables_keep_within_a_launch():
    """2^36 elements, and as many tensors as a table takes, have no more chunks than one launch."""
    one = dict(d_param=1 << 44, d_grad=1 << 45, d_m=1 << 46, d_v=1 << 47, d_m_scales=None, d_v_scales=None, d_copy=None,
               n=1 << 36, param_dtype=0, grad_dtype=0, state_dtype=0, weight_decay=0.0)
    assert R.rollout_adamw_table([R.AdamwTensor(*one.values())])[1] == 1 << 23
