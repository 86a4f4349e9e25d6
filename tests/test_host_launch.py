"""What the host side keeps between launches, without a GPU: the library runs in a child process under a stand-in for the
CUDA runtime (fake_cuda_runtime.cpp) that launches nothing."""
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2601_14327_gb300 import build as B

FAKE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "fake_cuda_runtime.cpp")


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    B.build()
    so = str(tmp_path_factory.mktemp("fake") / "libfake_cuda_runtime.so")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.nvcc()))), "include")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-I", inc, FAKE, "-o", so],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return so


def _child(fake, code, **env):
    head = """
        import ctypes, sys, threading
        from paper_2601_14327_gb300 import _lib as L
        fake = ctypes.CDLL(None)
        N = 1 << 20                   # stands for every device pointer: nothing reads it
        WS = dict(ws=N, ws_bytes=1 << 40, stream=1)
    """
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(head) + textwrap.dedent(code)], capture_output=True, text=True,
                       cwd=B.ROOT, env={**os.environ, "LD_PRELOAD": fake, **env}, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


CALLS = """
    def experts(T, d, E, k, F):
        R = L.moe_perm_rows_max(T, k, E)
        L.moe_grouped_ffn_fwd(N, N, E, d, F, R, N, N, N, N, N, **WS)
        L.moe_grouped_ffn_fwd_combine(N, N, E, d, F, R, N, N, N, N, T, k, N, N, N, N, N, **WS)
        L.moe_grouped_ffn_fwd_ckpt(N, N, E, d, F, R, N, N, N, N, N, N, **WS)
        L.moe_grouped_ffn_bwd_dgrad(N, N, N, E, d, F, R, N, N, N, None, N, N, T, k, N, N, N, **WS)
        L.moe_grouped_ffn_bwd_dgrad_ckpt(N, N, N, N, E, d, F, R, N, N, N, None, N, N, T, k, N, N, N, N, **WS)
        L.moe_grouped_ffn_bwd_wgrad(N, N, N, N, N, None, E, d, F, R, N, N, **WS)

    def gathered(T, d, E, k, F):
        R = L.moe_perm_rows_max(T, k, E)
        L.moe_grouped_ffn_fwd_gather(N, N, T, N, E, d, F, R, N, N, N, N, N, **WS)
        L.moe_grouped_ffn_bwd_wgrad_gather(N, N, N, T, N, N, N, None, E, d, F, R, N, N, **WS)

    def router(T, d, E, k):
        L.moe_route(N, N, None, None, T, d, E, k, None, None, N, N, N, **WS)
        L.moe_route_bwd(N, N, N, N, T, d, E, k, N, N, **WS)
        L.moe_route_bwd_dense(N, N, N, N, N, T, d, E, k, N, N, **WS)
        L.moe_route_dx(N, N, N, T, d, E, k, N, **WS)

    def balance(T, E, k, n_seq):
        L.moe_balance_loss(N, N, None, None, N, n_seq, T, E, k, 1.0, 1.0, N, N, N, N, N, **WS)
        L.moe_balance_loss_bwd(N, None, N, n_seq, T, E, k, 1.0, 1.0, N, N, N, None, N, stream=1)

    def everything():
        # one SM and CTA pairs, 128 and 256 columns, an odd last row block split off
        for s in ((40, 128, 4, 2, 128), (1021, 512, 32, 4, 384), (6000, 256, 4, 2, 256), (4100, 2048, 8, 4, 1408),
                  (66000, 128, 5, 4, 128), (66000, 1024, 5, 4, 512)):
            experts(*s)
        for s in ((1021, 512, 32, 4, 384), (16384, 4096, 16, 4, 2048)):
            gathered(*s)
        for s in ((1, 8, 1, 1), (1021, 512, 32, 4), (65536, 7168, 171, 8), (16384, 4096, 64, 8), (300, 264, 100, 4),
                  (32768, 4096, 256, 8), (5000, 1024, 130, 4)):
            router(*s)
        for s in ((37, 64, 6, 1), (65536, 256, 8, 24)):
            balance(*s)
"""


@pytest.mark.parametrize("first,second", [(0, 1), (1, 0)])
def test_every_entry_point_launches_on_a_second_device(fake, first, second):
    """What a kernel needs once is asked for once per device: after a process has used one, all calls work on another,
    with that one's number of co-resident CTA pairs."""
    out = _child(fake, CALLS + f"""
    for device in ({first}, {second}, {first}):
        fake.fake_use_device(device)
        everything()
        print(fake.fake_launches(), fake.fake_widest_cluster_grid() // 2, fake.fake_clusters(device))
    """)
    rows = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(rows) == 3 and rows[0][0] > 60
    for launches, pairs, room in rows:
        assert launches == rows[0][0] and pairs <= room, rows


def test_first_calls_from_two_threads(fake):
    """The first look-up of the driver's tensor-map call, still under way in another thread."""
    out = _child(fake, CALLS + """
    fake.fake_entry_point_ms(300)
    failed, gate = [], threading.Barrier(4)

    def call():
        try:
            gate.wait()
            L.moe_grouped_ffn_fwd(N, N, 4, 128, 128, 1024, N, N, N, N, N, **WS)
        except Exception as e:
            failed.append(repr(e))

    L.load()
    threads = [threading.Thread(target=call) for _ in range(4)]
    for t in threads: t.start()
    for t in threads: t.join()
    print(failed)
    """)
    assert out.strip() == "[]"
