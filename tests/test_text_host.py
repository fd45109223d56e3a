"""Host side of the text-model operators: what is refused, and how, before anything is launched.  No kernel runs."""
import ctypes
import math
import os
import random
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def S():
    from paper_2310_05674_b200 import build
    build.build()
    from paper_2310_05674_b200 import binding
    return binding


@pytest.fixture(scope="module")
def sizes(S, tmp_path_factory):
    """Answers of text_sizes.cpp, a line of numbers for each line asked."""
    from paper_2310_05674_b200 import build
    cuda = os.path.dirname(os.path.dirname(build.NVCC))
    exe = str(tmp_path_factory.mktemp("sizes") / "text_sizes")
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(cuda, "include"), "-I", os.path.join(ROOT, "include"),
                           "-I", build.CSRC, os.path.join(HERE, "text_sizes.cpp"), "-o", exe, S.LIB_PATH,
                           "-Wl,-rpath," + os.path.dirname(S.LIB_PATH), "-L", os.path.join(cuda, "lib64"), "-lcudart"])

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True).stdout
        rows = [[int(v) for v in line.split()] for line in out.splitlines()]
        assert len(rows) == len(lines)
        return rows
    return ask


@pytest.fixture
def blank():
    """Zeroed memory in the place of a context, for checks that come before anything in a context is looked at."""
    memory = ctypes.create_string_buffer(1 << 16)
    yield ctypes.addressof(memory)


@pytest.mark.parametrize("d", [2 ** 30 + 1, 2 ** 31 - 4, 2 ** 31 - 1])
def test_rows_that_32_bit_columns_cannot_step_through_are_refused(S, blank, d):
    assert S.lib.sama_embed(blank, S.SAMA_F32, 0, 1, d, 16, None, 1.0, None, None) == S.SAMA_ERR_SIZE
    assert S.lib.sama_embed_grad(blank, S.SAMA_F32, 0, 1, d, None, None, 1.0, -1, S.SAMA_F32, 1, 16, None) == S.SAMA_ERR_SIZE


def test_the_widest_row_is_accepted(S, blank):
    assert S.lib.sama_embed(blank, S.SAMA_F32, 0, 1, 2 ** 30, 16, None, 1.0, None, None) == S.SAMA_OK


def host_tensors(torch):
    """Every operand that is a tensor, by operator, on the host: each position is tried alone, beside plain addresses."""
    f, i, h = torch.zeros(64), torch.zeros(64, dtype=torch.int32), torch.zeros(64, dtype=torch.bfloat16)
    return {"sama_embed": ([0, 4, 4, 4], [f, i], [1.0], [f]),
            "sama_embed_grad": ([0, 4, 4, 4], [i, f], [1.0, -1, 0, 0], [f]),
            "sama_gated_ffn": ([1, 0, 4, 4, 4], [h] * 7, [], []),
            "sama_gated_ffn_grad": ([1, 0, 4, 4, 4], [h] * 11, [], [])}


@pytest.mark.parametrize("name,operands", [("sama_embed", 3), ("sama_embed_grad", 3), ("sama_gated_ffn", 7),
                                           ("sama_gated_ffn_grad", 11)])
def test_tensors_on_the_host_are_refused(S, name, operands):
    import torch
    for k in range(operands):
        n, a, between, b = host_tensors(torch)[name]
        a, b = ([t if at == k else 4096 * (at + 1) for at, t in part] for part in
                (list(enumerate(a)), list(enumerate(b, len(a)))))
        # (without a context, which is refused too, but later and with another status)
        with pytest.raises(S.SamaError) as e:
            getattr(S, name)(None, *n, *a, *between, *b, stream=0)
        assert e.value.status == S.SAMA_ERR_PARAM, k


def test_lists_of_tensors_on_the_host_are_refused(S):
    import torch
    for outs in (None, [None], [torch.zeros(8)]):
        with pytest.raises(S.SamaError) as e:
            S.TensorList([torch.zeros(8)], outs)
        assert e.value.status == S.SAMA_ERR_PARAM
    with pytest.raises(S.SamaError) as e:
        S.sama_clip_grads(None, S.TensorList([]), 1.0, torch.zeros(1), stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM


def test_tensors_on_another_gpu_than_the_context_are_refused(S, monkeypatch):
    class On:   # what the check looks at, of a tensor on GPU 1
        device = "cuda:1"

        def get_device(self):
            return 1

    monkeypatch.setitem(S._device_of, 4096, 0)
    with pytest.raises(S.SamaError) as e:
        S.sama_embed(4096, 0, 4, 4, 4, On(), 8192, 1.0, 16384, stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM
    tensors = S.TensorList([])
    tensors.device = 1
    with pytest.raises(S.SamaError) as e:
        S.sama_clip_grads(4096, tensors, 1.0, stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM


def test_a_list_in_place_takes_any_iterable(S):
    class OnGpu:
        dtype = device = None

        def numel(self):
            return 8

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 4096

    import torch
    OnGpu.dtype = torch.float32
    x = OnGpu()
    tensors = S.TensorList(t for t in [x, x])
    assert tensors.ins == tensors.outs == [x, x] and tensors.c()[1].out == tensors.c()[1].in_ == 4096


def embed_line(n, vocab, d, dtype=1, grad_dtype=0, shift=0):
    return "embed %d %d %d %d %d %d %d" % (dtype, n, vocab, d, 4096 + (4 if dtype == 0 else 2) * shift, grad_dtype, 8192)


def test_no_smaller_embedding_gradient_needs_a_larger_workspace(sizes):
    """What a call reserves covers every call of at most its sizes, of any type and alignment."""
    # fewer tokens have shorter pieces, and more parts
    at = {n: sizes([embed_line(n, 50021, 1024)])[0] for n in (14000, 14192, 16384, 28416)}
    assert at[14192][1] > at[16384][1] > at[28416][1]          # (what the plans need)
    assert at[14000][0] <= at[14192][0] <= at[16384][0] <= at[28416][0]
    rng = random.Random(3)

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    asked = []
    for _ in range(4000):
        n, vocab, d = log(1, 1 << 21), log(1, 1 << 25), log(1, 1 << 18 if rng.random() < 0.2 else 8192)
        if rng.random() < 0.3:
            n, d = rng.choice([n, 2047, 2048, 2049, 131072]), rng.choice([d, 8, 32, 33, 128, 256, 1024, 129152, 129153])
        asked.append((n, vocab, d))
        asked.append(tuple(max(1, v if rng.random() < 0.4 else int(v * rng.random())) for v in (n, vocab, d)))
    kinds = [(dt, gt, shift) for dt, gt in ((0, 0), (1, 0), (1, 1), (2, 0), (2, 2)) for shift in (0, 1)]
    rows = sizes([embed_line(*a, *k) for a in asked for k in kinds])
    for i in range(0, len(asked), 2):
        large, small = (rows[j * len(kinds):(j + 1) * len(kinds)] for j in (i, i + 1))
        assert len({r[0] for r in large}) == 1                 # not by type, not by alignment
        assert small[0][0] <= large[0][0], asked[i:i + 2]
        assert all(need <= reserved for reserved, need in large + small), asked[i:i + 2]


def test_the_feed_forward_block_reserves_what_it_uses(sizes):
    """H (three such matrices for a backward pass), and the operands that are copied: rows of whole 16-byte groups."""
    def group(x):
        return -(-x // 8) * 8

    def area(rows, cols):
        return -(-rows * group(cols) * 2 // 256) * 256

    d, f = 3429, 9421
    weights = 2 * area(f, d) + area(d, f)
    for n in (1, 16, 17, 700):
        hidden, x = area(n, f), area(n, d)
        got = [r[0] for r in sizes(["ffn %d %d %d %d %d" % (n, d, f, grad, copies) for grad in (0, 1) for copies in (0, 1)])]
        # up to 16 tokens, the forward pass reads odd operands where they are
        assert got == [hidden, hidden + (x + weights if n > 16 else 0), 3 * hidden, 5 * hidden + 2 * x + weights], n


def test_no_memory_for_the_set_up_has_its_own_status(S, sizes):
    """Error 2 is cudaErrorMemoryAllocation; 1, 719 and 900 are other errors (value, launch, capture)."""
    assert sizes(["setup %d" % e for e in (2, 1, 719, 900)]) == [
        [S.SAMA_ERR_NOMEM, 2], [S.SAMA_ERR_CUDA, 1], [S.SAMA_ERR_CUDA, 719], [S.SAMA_ERR_CUDA, 900]]


def test_only_weights_are_read_through_the_read_only_path():
    """A kernel of the text-model operators may start before the launch whose results it reads has ended, and may write
    what it has read (clipping in place).  Neither goes with loads that promise that the data does not change while the
    kernel runs: __ldg, ld.global.nc, and pointers to const that are declared to have no alias."""
    csrc = os.path.join(ROOT, "paper_2310_05674_b200", "csrc")
    found = {}
    for f in ("clip_grads.cu", "embed.cu", "gated_ffn.cu", "num_types.h"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read())
        found[f] = len(re.findall(r"__ldg\b|ld\.global\.nc|const\s+\w+\s*\*\s*__restrict__", text))
    assert found == {"clip_grads.cu": 0, "embed.cu": 0, "gated_ffn.cu": 1, "num_types.h": 0}   # load_weights
