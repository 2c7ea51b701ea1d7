"""Host plan of the attention over shared prefixes (CPU): a C++ program compiled
against the built library (tests/native/shared_plan_check.cpp) checks what the
kernels index from it, over the measured batches, edges of the tables and random
batches; and the refusals of the two entry points."""
import os
import random
import shutil
import subprocess

import pytest

from test_boundary_cpu import ppas  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2608_15171_gb300")


@pytest.fixture(scope="module")
def checker(ppas, tmp_path_factory):  # noqa: F811
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("splan") / "shared_plan_check")
    cmd = [gxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
           "-I", "/usr/local/cuda/include", os.path.join(ROOT, "tests", "native", "shared_plan_check.cpp"),
           "-o", exe, "-L", PKG, "-lppas", f"-Wl,-rpath,{PKG}", "-L/usr/local/cuda/lib64", "-lcudart"]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return exe


def _run(exe, cases, sms=152):
    text = "".join(f"{sms} {hq} {hk} {len(rows)} " + " ".join(f"{r} {p}" for r, p in zip(rows, pre)) + " " +
                   " ".join(map(str, ctx)) + "\n" for hq, hk, rows, pre, ctx in cases)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for line, case in zip(out, cases):
        assert line.startswith("ok "), (line, case[:4])
    return [[int(x) for x in line.split()[1:]] for line in out]


def _batch(rng, hq, hk, rows, pre, lo, hi):
    ctx = [max(1, p + rng.randint(lo, hi)) for n, p in zip(rows, pre) for _ in range(n)]
    return hq, hk, rows, pre, ctx


@pytest.mark.parametrize("sms", [152, 148, 132, 1, 256])
def test_batches_and_edges(checker, sms):
    rng = random.Random(1)
    cases = [_batch(rng, *c) for c in [
        (16, 2, [4], [2048], 1, 64), (16, 2, [32], [24992], 17, 500), (32, 8, [64], [30000], 1, 1000),
        (16, 2, [9, 33, 1, 21, 6], [4096, 25008, 9984, 512, 0], 1, 300),
        (16, 2, [1], [0], 1, 1), (16, 2, [1], [25008], 1, 1), (8, 8, [2], [16], 0, 0), (8, 8, [1], [16], 0, 0),
        (32, 8, [512], [128], 0, 40), (32, 8, [513], [256], 1, 1), (16, 2, [2000], [1024], 1, 20),
        (8, 8, [1] * 300, [64] * 300, 1, 9), (8, 8, [2] * 200, [128] * 200, 1, 9),
        (256, 256, [512], [1000 * 16], 1, 2), (512, 256, [40, 500], [65536, 65552], 1, 2),
        (512, 64, [512], [4096], 1, 2), (16, 2, [300], [65535 * 128], 0, 0), (8, 4, [3], [65535 * 128 - 4096], 1, 4096),
        (64, 32, [100], [40 * 65536], 1, 5), (16, 2, [5], [0], 8000000, 8388480), (16, 2, [1], [0], 8388480, 8388480),
    ]]
    _run(checker, cases, sms)


def test_random_batches(checker):
    rng = random.Random(2)
    cases = []
    for _ in range(400):
        hq, hk = rng.choice([(16, 2), (32, 8), (8, 4), (8, 8), (4, 1), (64, 8), (16, 16)])
        n = rng.choice([1, 1, 2, 5, 40])
        rows = [rng.choice([1, 2, 3, rng.randint(1, 70)]) for _ in range(n)]
        pre = [rng.choice([0, 16, 16 * rng.randint(1, 2000)]) for _ in range(n)]
        cases.append(_batch(rng, hq, hk, rows, pre, rng.choice([0, 1]), rng.choice([1, 16, 2000])))
    for sms in (152, 132):
        _run(checker, cases, sms)


def test_one_round_of_pieces(checker):
    """The measured batches' pieces and own keys fill one round of the SMs."""
    rng = random.Random(3)
    for got in _run(checker, [_batch(rng, 16, 2, [32], [24992], 17, 500), _batch(rng, 32, 8, [64], [30000], 1, 1000),
                              _batch(rng, 16, 2, [4], [2048], 1, 64)]):
        launches, pieces, items, own_ctas = got[:4]
        assert launches == 1 and pieces + own_ctas <= 152


def test_refusals(ppas):  # noqa: F811
    ok = dict(q=16, k_cache=16, v_cache=16, num_blocks=4, d_block_tables=16, max_blocks_per_seq=4, ctx_lens=[40, 33],
              group_rows=[2], prefix_lens=[32], n_q_heads=16, n_kv_heads=2, head_dim=128, scale=0.1, out=16,
              workspace=256, workspace_bytes=1 << 40, stream=0)

    def status(**kw):
        with pytest.raises(ppas.PpasError) as e:
            ppas.ppas_shared_attention_step(**{**ok, **kw})
        return e.value.status

    for kw in (dict(ctx_lens=[40]), dict(group_rows=[3]), dict(group_rows=[0, 2], prefix_lens=[0, 0]),
               dict(prefix_lens=[31]), dict(prefix_lens=[-16]), dict(ctx_lens=[40, 31]), dict(ctx_lens=[40, 65]),
               dict(prefix_lens=[0], ctx_lens=[40, 0]), dict(n_q_heads=15), dict(n_kv_heads=0), dict(q=0), dict(q=8),
               dict(out=0), dict(out=24), dict(k_cache=8), dict(v_cache=0), dict(d_block_tables=0), dict(num_blocks=0),
               dict(scale=0.0), dict(scale=float("nan")), dict(head_dim=0), dict(workspace=128)):
        assert status(**kw) == ppas.PPAS_ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=64), dict(n_q_heads=12, n_kv_heads=1), dict(n_q_heads=1024, n_kv_heads=128),
               dict(ctx_lens=[40, 65535 * 128 + 1], max_blocks_per_seq=65535 * 8 + 1),
               dict(n_q_heads=64, n_kv_heads=64, prefix_lens=[21 * 65536], ctx_lens=[21 * 65536] * 2,
                    max_blocks_per_seq=21 * 4096)):
        assert status(**kw) == ppas.PPAS_ERR_UNSUPPORTED, kw
    assert status(workspace_bytes=255) == ppas.PPAS_ERR_CAPACITY
    assert status(workspace=None) == ppas.PPAS_ERR_CAPACITY
    ppas.ppas_shared_attention_step(**{**ok, "group_rows": [], "prefix_lens": [], "ctx_lens": [], "q": 0})  # no-op
    assert ppas.ppas_shared_attention_workspace_size([], [], [], 16, 2) == 0
    assert ppas.ppas_shared_attention_workspace_size([40, 33], [2], [31], 16, 2) == 0
    a = ppas.ppas_shared_attention_workspace_size([25010, 25020], [2], [24992], 16, 2)
    assert a > 0 and a % 256 == 0 and a == ppas.ppas_shared_attention_workspace_size([25010, 25020], [2], [24992], 16, 2)
