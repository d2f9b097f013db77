"""The learning calls' host code without a GPU: networks.cpp linked with the stand-in runtime
(tests/shim/fake_hip.cpp) and launchers that write down what they are given (tests/shim/fake_learn.cpp), for
which buffers a call uses, keeps and replaces."""

import ctypes as C
import gc
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2608_27612_amd import emr as E
from paper_2608_27612_amd import workloads as W

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2608_27612_amd", "csrc")
FLAGS = ["g++", "-std=c++17", "-O1", "-fPIC", "-w", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include"]
FIELDS = ("step", "items", "joins", "step_items", "values", "partial", "state", "count", "first", "at")
MB = 1 << 20


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    at = tmp_path_factory.mktemp("fake")
    path, plain = str(at / "libfake.so"), str(at / "fake_hip.o")
    subprocess.check_call(FLAGS + ["-Demr_launch_net=emr_launch_net_of_no_kernel", "-DhipEventRecord=plain_hipEventRecord",
                                   "-DhipEventSynchronize=plain_hipEventSynchronize", "-c",
                                   os.path.join(HERE, "shim", "fake_hip.cpp"), "-o", plain])
    subprocess.check_call(FLAGS + ["-shared", "-Wl,-Bsymbolic", plain, os.path.join(HERE, "shim", "fake_learn.cpp")]
                          + [os.path.join(CSRC, s) for s in ("runtime.cpp", "networks.cpp", "plan.cpp", "pack.cpp",
                                                             "sched.cpp", "jit.cpp", "record_file.cpp")]
                          + ["-o", path])
    return path


@pytest.fixture
def lib(built, tmp_path):
    """The binding on a copy of the stand-in library, and the stand-in's own calls."""
    path = str(tmp_path / "libfake.so")
    shutil.copy(built, path)
    keep = E._lib, E.LIB_PATH
    E._lib, E.LIB_PATH = None, path
    L = E.lib()
    for name, (res, args) in {"fake_capturing": (None, [C.c_int]), "fake_held": (C.c_int64, []),
                              "fake_hold_events": (None, [C.c_int]), "fake_counts": (None, [C.c_void_p]),
                              "fake_size": (C.c_int64, [C.c_void_p]), "fake_launches": (C.c_int64, []),
                              "fake_launch": (None, [C.c_int64, C.c_void_p]),
                              "fake_sums": (C.c_int64, [C.c_int64, C.c_int64]),
                              "fake_light_edges": (C.c_uint32, [C.c_uint32, C.c_uint32])}.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    yield L
    gc.collect()
    E._lib, E.LIB_PATH = keep


def launches(lib, first=0):
    out = []
    for i in range(first, lib.fake_launches()):
        v = (C.c_int64 * len(FIELDS))()
        lib.fake_launch(i, v)
        out.append(dict(zip(FIELDS, v)))
    return out


def networks(nodes, edges):
    """A handle of genomes of one input, one output, and these numbers of nodes and edges (spread evenly over
    the nodes but the input, from node 0 on)."""
    src = W.sources_array([(0.0, -1.0, 0), (0.0, 1.0, 1)])
    node_offset, degrees, ins = [0], [], []
    for n, e in zip(nodes, edges):
        d = np.full(n, e // (n - 1))
        d[0] = 0
        d[1] += e - d.sum()
        degrees.append(d)
        ins.append(node_offset[-1] + np.arange(e) % n)
        node_offset.append(node_offset[-1] + n)
    in_offset = np.concatenate([[0], np.cumsum(np.concatenate(degrees))]).astype(np.int64)
    ins = np.concatenate(ins).astype(np.uint32)
    w = np.zeros(len(ins), np.float32)
    node_offset = np.array(node_offset, np.int64)
    h = C.c_void_p()
    assert E.lib().emr_load_networks(src.ctypes.data, 2, 0, len(nodes), node_offset.ctypes.data, None,
                                     in_offset.ctypes.data, ins.ctypes.data, w.ctypes.data, C.byref(h), None) == 0
    return h


ANY = 1 << 20  # an aligned address that nothing reads
ANY_W = np.zeros(1000, np.float32)


def keep(h, patterns, steps=3):
    return E.lib().emr_activate_keep(h, ANY, patterns, steps, ANY, ANY, 1 << 50, None)


def back(h, patterns, steps=3):
    return E.lib().emr_activate_backward(h, ANY, patterns, steps, ANY, ANY, 1 << 50, ANY, ANY, None, None)


def buffers(logged):
    return {l[k] for l in logged for k in ("items", "joins", "step_items", "values", "partial", "state") if l[k]}


# one genome that is stepped at 64 patterns and not at 96, among smaller ones
STEPPED = ([1000] + [200] * 100, [100000] + [9000] * 100)


def contents(lib, p):
    return C.string_at(p, min(lib.fake_size(p), MB))


@pytest.mark.parametrize("later", ["fewer patterns", "more patterns", "many numbers of patterns"])
def test_what_a_captured_call_uses_stays(lib, later):
    """A captured call names its tables and buffers in every replay: no later call on the handle replaces or
    rewrites them, whether it needs larger ones (which calls on fewer patterns may) or leaves more than 64
    numbers of patterns behind, and none serves another handle."""
    h = networks(*STEPPED)
    for f in (keep, back):
        assert f(h, 96) == 0, lib.emr_last_error()
    at = lib.fake_launches()
    lib.fake_capturing(1)
    for f in (keep, back):
        assert f(h, 96) == 0, lib.emr_last_error()
    lib.fake_capturing(0)
    used = buffers(launches(lib, at))
    tables = {l[k] for l in launches(lib, at) for k in ("items", "joins", "step_items") if l[k]}
    assert len(used) >= 5
    was = {p: contents(lib, p) for p in tables}
    for patterns in {"fewer patterns": [64], "more patterns": [3000],
                     "many numbers of patterns": range(1, 80)}[later]:
        for f in (keep, back):
            assert f(h, patterns) == 0, lib.emr_last_error()
    other = networks(*STEPPED)
    at = lib.fake_launches()
    for patterns in (96, 64, 20):
        for f in (keep, back):
            assert f(other, patterns) == 0, lib.emr_last_error()
    assert not used & buffers(launches(lib, at))
    for p in used & tables:
        assert contents(lib, p) == was[p]
    # and the same call again names the same tables
    at = lib.fake_launches()
    assert keep(h, 96) == 0 and back(h, 96) == 0
    assert {l[k] for l in launches(lib, at) for k in ("items", "joins", "step_items") if l[k]} == tables
    for x in (other, h):
        lib.emr_free_networks(x)


def test_states_that_a_captured_activation_uses_stay(lib):
    """emr_activate's stepwise states, and the kept activation's of genomes larger than a workgroup's memory,
    are one buffer of the handle."""
    h = networks([20000], [19999])
    x = np.zeros((8, 1), np.float32)
    for capture in (0, 1):
        lib.fake_capturing(capture)
        at = lib.fake_launches()
        assert lib.emr_activate(h, x.ctypes.data, 8, 2, ANY, None) == 0
    lib.fake_capturing(0)
    used = {l["state"] for l in launches(lib, at) if l["step"] == 9}
    assert len(used) == 1
    assert keep(h, 100) == 0
    other = networks([20000], [19999])
    at = lib.fake_launches()
    assert lib.emr_activate(other, x.ctypes.data, 8, 2, ANY, None) == 0
    assert not used & buffers(launches(lib, at))
    for v in (other, h):
        lib.emr_free_networks(v)


def test_a_capture_that_would_need_new_buffers_is_refused(lib):
    """Under capture a call lays nothing out and allocates nothing: it is refused, with nothing enqueued, until
    the same call has run once."""
    h = networks(STEPPED[0] + [20000], STEPPED[1] + [30000])
    lib.fake_capturing(1)
    for f in (keep, back):
        held, at = lib.fake_held(), lib.fake_launches()
        assert f(h, 96) == E.EMR_E_DEVICE
        assert b"capture" in lib.emr_last_error()
        assert (lib.fake_held(), lib.fake_launches()) == (held, at)
    lib.fake_capturing(0)
    assert keep(h, 96) == 0
    lib.fake_capturing(1)
    held, at = lib.fake_held(), lib.fake_launches()
    assert keep(h, 97) == E.EMR_E_DEVICE  # another number of patterns
    assert back(h, 96) == E.EMR_E_DEVICE  # the derivatives' buffers
    assert (lib.fake_held(), lib.fake_launches()) == (held, at)
    lib.fake_capturing(0)
    assert back(h, 96) == 0
    lib.fake_capturing(1)
    assert keep(h, 96) == 0 and back(h, 96) == 0
    lib.fake_capturing(0)
    lib.emr_free_networks(h)


def test_the_plan_in_use_stays_among_many(lib):
    """Of more than 64 numbers of patterns, the one used longest ago is laid out anew, not the oldest."""
    h = networks([30], [100])
    out = (C.c_int32 * 3)()
    for patterns in range(1, 120):
        assert keep(h, patterns) == 0
        lib.fake_counts(out)
        waits = out[0]
        assert keep(h, 1) == 0
        lib.fake_counts(out)
        assert out[0] == waits
    lib.emr_free_networks(h)


def test_weights_set_by_a_graph_captured_before_the_layout(lib):
    """The layouts hold copies of the weights. A graph captured before there were any sets the handle's
    weights alone, in every replay: the learning calls of that handle then copy them anew."""
    for first in ("captured", "eager"):
        h = networks([30, 40], [100, 90])
        lib.fake_capturing(first == "captured")
        assert lib.emr_networks_set_weights(h, ANY_W.ctypes.data, None) == 0
        lib.fake_capturing(0)
        for f in (keep, back, keep):
            at = lib.fake_launches()
            assert f(h, 20) == 0
            steps = [l["step"] for l in launches(lib, at)]
            assert (23 in steps) == (first == "captured")
            assert 23 not in steps or steps.index(23) < steps.index(25 if f is back else 24)
        lib.emr_free_networks(h)


def test_a_freed_handle_waits_for_the_calls_before_a_capture(lib):
    """The handle's buffers go back to the cache once the last call that ran has ended, whatever was captured
    after it (an event recorded into a graph cannot be waited for)."""
    h = networks([30], [100])
    assert keep(h, 5) == 0
    lib.fake_hold_events(1)
    assert keep(h, 5) == 0
    lib.fake_capturing(1)
    assert keep(h, 5) == 0
    lib.fake_capturing(0)
    out = (C.c_int32 * 3)()
    lib.fake_counts(out)
    waits = out[0]
    lib.emr_free_networks(h)
    lib.fake_counts(out)
    assert out[0] == waits + 1
    lib.fake_hold_events(0)


@pytest.mark.parametrize("nodes,edges,patterns", [
    ([4000] * 40, [240000] * 40, 10000), ([4000] * 40, [240000] * 40, 65536), ([773] * 150, [40000] * 150, 65536),
    ([5000], [20000000], 65536), ([5000], [20000000], 600), ([1000] + [200] * 100, [100000] + [9000] * 100, 64)])
def test_workspaces_have_a_bound(lib, nodes, edges, patterns):
    """The gradients' partial sums and the states outside LDS take 2 GiB and a copy of the genomes' own at most
    (the states of genomes with a launch for each step: three float arrays), however many patterns there are."""
    h = networks(nodes, edges)
    at = lib.fake_launches()
    assert back(h, patterns) == 0, lib.emr_last_error()
    logged = launches(lib, at)
    partial, = {l["partial"] for l in logged if l["partial"]}
    one = sum(4 * lib.fake_sums(n, e) for n, e in zip(nodes, edges))
    values = sum(3 * 4 * n * -(-patterns // 32) * 32 + 2 * 16 * 8 * (n + 1) for n in nodes)
    # (the stand-in hands out whole pages, the cache buffers of up to twice the size)
    assert 0 < lib.fake_size(partial) <= (2 << 30) + one + 4096
    if any(l["step"] == 32 for l in logged):
        v, = {l["values"] for l in logged if l["step"] == 32}
        assert lib.fake_size(v) <= values + (2 << 30) + 4096
    assert sum(l["count"] for l in logged if l["step"] in (25, 32)) >= 256 or patterns < 256
    lib.emr_free_networks(h)


def places(degrees, light_edges):
    """Places of one layout by source (rows of these numbers of edges), as the slices' kernel lays it out."""
    d = np.sort(np.asarray(degrees))[::-1]
    light = light_edges(int(d.sum()), len(d))
    heavy, rest = d[d > light], d[d <= light]
    four = lambda v: -(-v // 4) * 4  # noqa: E731
    return int((16 * four(-(-heavy // 16))).sum() + sum(16 * four(int(rest[i])) for i in range(0, len(rest), 16)))


@pytest.mark.parametrize("seed", range(200))
def test_an_items_sums_hold_both_layouts(lib, seed):
    """Rows of even, falling, few and single hub degrees, around the borders of the light rows."""
    rng = np.random.default_rng(seed)
    sets = []
    for _ in range(2):
        n = int(np.exp(rng.uniform(0, np.log(3000))))
        kind = rng.integers(0, 6)
        if kind == 0:
            d = rng.integers(0, rng.choice([2, 20, 70, 2000]), n)
        elif kind == 1:
            d = np.minimum(rng.pareto(rng.uniform(0.3, 2.0), n) * 10, 10000).astype(int)
        elif kind == 2:
            d = np.zeros(n, int)
            d[: max(1, n // 100)] = rng.choice([65, 66, 1021, 1022, 5000])
        elif kind == 3:
            d = np.full(n, rng.choice([0, 1, 4, 5, 64, 65, 300, 1021, 1022, 1025]))
        elif kind == 4:
            d = np.where(np.arange(n) % 16 == 0, rng.choice([17, 64, 65, 400]), rng.choice([0, 1, 16, 64]))
        else:
            d = np.where(rng.random(n) < 0.25, 65, 16)
        sets.append(d)
    n, e = sum(len(d) for d in sets), int(sum(d.sum() for d in sets))
    assert sum(places(d, lib.fake_light_edges) for d in sets) <= lib.fake_sums(n, e)


@pytest.mark.parametrize("rows,n", [(1, 1), (1, 4), (2, 3), (5, 1), (4, 3), (7, 2)])
def test_a_gradient_over_the_scores_is_theirs_row_by_row(lib, rows, n):
    """Every place of the gradient's rows beside the scores' (in entries): refused where an entry of the two is the
    same one, but for rows that lie on each other. (No kernel runs.)"""
    x = 1 << 20
    for type, size in ((E.EMR_F32, 4), (E.EMR_BF16, 2)):
        for stride in (0, 1, n - 1, n, n + 1, 2 * n, 2 * n + 1, 3 * n):
            scores = E.emr_scores(x, type, rows, n, stride)
            mine = {r * stride + k for r in range(rows) for k in range(n)}
            for grad_stride in (n, n + 1, 2 * n, 3 * n):
                rest = {r * grad_stride + k for r in range(rows) for k in range(n)}
                for d in range(-3 * n * rows - 2, 3 * n * rows + 3):
                    st = lib.emr_answer_loss(C.byref(scores), ANY, None, C.c_float(1.0), ANY, x + d * size,
                                             grad_stride, None)
                    same = d == 0 and (rows == 1 or stride == grad_stride)
                    fits = same or not any(k - d in rest for k in mine)
                    assert st == (E.EMR_OK if fits else E.EMR_E_INVAL), (stride, grad_stride, d)
