"""Activation that keeps its states in 8 bits, and the gradients from them, against 64-bit arithmetic
over the same edges and codes: loaded and built networks, pattern counts around every block size, networks
of no, few and very many nodes and edges, one step and many, self-connections and cycles."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_27612_amd import workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_27612_amd import emr as m
    return m


def substrate(n_in, n_out, mixed=False):
    """Inputs, then outputs; mixed: every other one, as far as they reach."""
    ins = [(i * 0.01, -1.0, 0) for i in range(n_in)]
    outs = [(i * 0.01, 1.0, 1) for i in range(n_out)]
    if not mixed:
        return W.sources_array(ins + outs)
    both = [v for pair in zip(outs, ins) for v in pair]
    k = min(n_in, n_out)
    return W.sources_array(both + ins[k:] + outs[k:])


def random_nets(seed, hidden, n_in, n_out, degree, mixed=False, empty=()):
    """Flat arrays of genomes with these numbers of hidden nodes: every hidden and output node has up to
    `degree` incoming edges from any node (itself, outputs and inputs too); the genomes in `empty` have none."""
    rng = np.random.default_rng(seed)
    subs = substrate(n_in, n_out, mixed)
    is_in = np.array([int(s["dir"]) == 0 for s in subs])
    node_offset, in_offset, src, w = [0], [0], [], []
    for g, m in enumerate(hidden):
        n = n_in + n_out + m
        base = node_offset[-1]
        for i in range(n):
            d = 0
            if not (i < len(is_in) and is_in[i]) and g not in empty:
                d = int(rng.integers(0, min(degree, n) + 1))
                if i < len(is_in) and rng.random() < 0.7:
                    d = min(n, 4 * degree)
            s = np.sort(rng.choice(n, d, replace=False)) if d else np.zeros(0, int)
            src.append(base + s)
            w.append(rng.standard_normal(d) * 2 / np.sqrt(max(d, 1)))
            in_offset.append(in_offset[-1] + d)
        node_offset.append(base + n)
    return {"subs": subs, "is_in": is_in, "node_offset": np.array(node_offset),
            "in_offset": np.array(in_offset), "src": np.concatenate(src).astype(np.int64),
            "w": np.concatenate(w).astype(np.float32)}


def load(emr, a):
    return emr.emr_load_networks(a["subs"], a["node_offset"], a["in_offset"], a["src"], a["w"])


def from_handle(emr, net, subs):
    i = net.info()
    get = lambda p, n, d: emr._dev_to_host(p, n, d)  # noqa: E731
    return {"subs": subs, "is_in": np.array([int(s["dir"]) == 0 for s in subs]),
            "node_offset": get(i.node_offset, i.n_genomes + 1, np.int64),
            "in_offset": get(i.in_offset, i.nodes + 1, np.int64),
            "src": get(i.in_src, i.edges, np.uint32).astype(np.int64),
            "w": get(i.in_w, i.edges, np.float32)}


def forward64(a, x, steps):
    """Per step (after it) the states of all nodes [nodes, patterns], float64."""
    n_in, n_sub = int(a["is_in"].sum()), len(a["is_in"])
    nodes = int(a["node_offset"][-1])
    s = np.zeros((nodes, len(x)))
    held = np.concatenate([o + np.nonzero(a["is_in"])[0] for o in a["node_offset"][:-1]])
    s[held] = np.tile(x.T, (len(a["node_offset"]) - 1, 1))
    assert s[held].shape[0] == n_in * (len(a["node_offset"]) - 1) and n_sub >= n_in
    dst = np.repeat(np.arange(nodes), np.diff(a["in_offset"]))
    out = [s]
    for _ in range(steps):
        z = np.zeros_like(s)
        if len(dst):
            first = np.unique(dst, return_index=True)
            z[first[0]] = np.add.reduceat(a["w"].astype(np.float64)[:, None] * s[a["src"]], first[1], axis=0)
        s = 1.0 / (1.0 + np.exp(-z))
        s[held] = out[0][held]
        out.append(s)
    return out


def output_nodes(a):
    return a["node_offset"][:-1, None] + np.nonzero(~a["is_in"])[0]


def backward64(a, x, steps, outputs, codes, grad_out):
    """(grad_w, grad_x, and for each the sum of the terms' sizes), float64, from the codes
    [steps - 1, nodes, patterns]."""
    G, P = len(a["node_offset"]) - 1, len(x)
    nodes = int(a["node_offset"][-1])
    held = np.concatenate([o + np.nonzero(a["is_in"])[0] for o in a["node_offset"][:-1]])
    dst = np.repeat(np.arange(nodes), np.diff(a["in_offset"]))
    src, w = a["src"], a["w"].astype(np.float64)
    gw, gx = np.zeros(len(src)), np.zeros((len(held), P))
    aw, ax = np.zeros(len(src)), np.zeros((len(held), P))
    gz, az = np.zeros((nodes, P)), np.zeros((nodes, P))
    at = output_nodes(a).reshape(-1)
    o = outputs.astype(np.float64).transpose(0, 2, 1).reshape(-1, P)
    if steps:
        gz[at] = grad_out.astype(np.float64).transpose(0, 2, 1).reshape(-1, P) * o * (1 - o)
        az = np.abs(gz)
    for t in range(steps, 0, -1):
        s = codes[t - 2].astype(np.float64) / 255 if t > 1 else np.zeros((nodes, P))
        s[held] = np.tile(x.T, (G, 1))
        gw += (gz[dst] * s[src]).sum(1)
        aw += (az[dst] * np.abs(s[src])).sum(1)
        d, b = np.zeros((nodes, P)), np.zeros((nodes, P))
        np.add.at(d, src, w[:, None] * gz[dst])
        np.add.at(b, src, np.abs(w)[:, None] * az[dst])
        gx += d[held]
        ax += b[held]
        gz, az = d * s * (1 - s), b * s * (1 - s)
        gz[held] = 0
        az[held] = 0
    n_in = int(a["is_in"].sum())
    back = lambda v: v.reshape(G, n_in, P).transpose(0, 2, 1)  # noqa: E731
    return gw, back(gx), aw, back(ax)


def unit(steps, terms):
    """Relative error, against the sum of the terms' sizes, of `steps` steps backwards and a sum of products:
    in each step a sum of at most `terms` products (each in a chain of at most terms fused adds) and
    five roundings for the factor s (1 - s), the code's scale and the store."""
    return (steps * (terms + 8) + terms + 8) * 2.0 ** -24


def check(emr, net, a, x, steps, seed=0, codes=None):
    """Forward: outputs within the sums' rounding of the float64 states and of emr_activate's, codes within
    half a step more; backward against float64 from the library's codes."""
    xd = torch.tensor(x, dtype=torch.float32, device="cuda")
    x = xd.cpu().numpy().astype(np.float64)
    out, kept = net.activate_keep(xd, steps)
    states = forward64(a, x, steps)
    held = np.concatenate([o + np.nonzero(a["is_in"])[0] for o in a["node_offset"][:-1]])
    got = kept.values().cpu().numpy()
    assert got.shape == (max(steps - 1, 0), int(a["node_offset"][-1]), len(x))
    deg = int(np.diff(a["in_offset"]).max()) if len(a["in_offset"]) > 1 else 0
    big = np.bincount(np.repeat(np.arange(len(a["in_offset"]) - 1), np.diff(a["in_offset"])),
                      weights=np.abs(a["w"]), minlength=1).max() if len(a["w"]) else 0.0
    # one step's error: a sum of |w| <= big in a chain of up to deg adds, slope 1 / 4, and the sigmoid's; the
    # error of the states before it grows by big / 4 a step
    one = big * (deg + 8) * 2.0 ** -24 / 4 + 2.0 ** -22
    slack = sum(one * max(1.0, big / 4) ** k for k in range(steps))
    want = states[-1][output_nodes(a)].transpose(0, 2, 1)
    assert np.abs(out.cpu().numpy() - want).max() <= slack + 1e-7
    assert np.abs(out.cpu().numpy() - net.activate(x, steps)).max() <= 2 * slack + 1e-7
    for t in range(steps - 1):
        want = states[t + 1].copy()
        want[held] = 0
        assert np.abs(got[t] - want).max() <= 0.5 / 255 + slack + 1e-7
        assert (got[t][held] == 0).all()
    i = net.info()
    rng = np.random.default_rng(seed)
    grad_out = (rng.standard_normal((i.n_genomes, len(x), i.n_outputs)) / len(x)).astype(np.float32)
    if codes is not None:
        kept = emr.kept_from_codes(torch.tensor(codes, device="cuda"))
    gw, gx = net.activate_backward(xd, steps, out, kept, torch.tensor(grad_out, device="cuda"),
                                   grad_inputs=True)
    gw2, none = net.activate_backward(xd, steps, out, kept, torch.tensor(grad_out, device="cuda"))
    assert none is None and torch.equal(gw, gw2)
    c = np.rint(kept.values().double().cpu().numpy() * 255)
    ww, wx, aw, ax = backward64(a, x, steps, out.cpu().numpy(), c, grad_out)
    terms = int(max(deg, len(x), np.bincount(a["src"]).max() if len(a["src"]) else 0))
    eps = unit(steps, terms)
    assert (np.abs(gw.cpu().numpy() - ww) <= eps * aw + 1e-30).all()
    assert (np.abs(gx.cpu().numpy() - wx) <= eps * ax + 1e-30).all()
    return gw, gx


@pytest.mark.parametrize("patterns", [1, 3, 4, 5, 8, 9, 16, 17, 33, 100])
def test_pattern_counts(emr, patterns):
    a = random_nets(1, [0, 1, 2, 5, 17, 40, 130], 3, 2, 9)
    net = load(emr, a)
    x = np.random.default_rng(patterns).uniform(-1, 1, (patterns, 3))
    check(emr, net, a, x, 4)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 7, 20])
def test_steps(emr, steps):
    a = random_nets(2, [3, 0, 60, 200], 5, 3, 12, mixed=True)
    net = load(emr, a)
    check(emr, net, a, np.random.default_rng(steps).uniform(-1, 1, (21, 5)), steps)


@pytest.mark.parametrize("hidden", [[], [0], [1], [0, 0, 0], [300], [600], [800, 3], [1200, 0, 7], [2500], [6000, 40]])
def test_sizes(emr, hidden):
    if not hidden:
        with pytest.raises(emr.EmrError):
            emr.emr_load_networks(substrate(1, 1), [0], [0], [], [])
        return
    a = random_nets(len(hidden) + sum(hidden), hidden, 2, 1, 20)
    net = load(emr, a)
    for patterns in (2, 19):
        check(emr, net, a, np.random.default_rng(3).uniform(-1, 1, (patterns, 2)), 3)


def test_no_edges_and_empty_genomes(emr):
    a = random_nets(5, [4, 9, 0, 30], 2, 2, 8, empty=(0, 2))
    net = load(emr, a)
    check(emr, net, a, np.random.default_rng(3).uniform(-1, 1, (5, 2)), 3)
    a = random_nets(5, [4, 9], 2, 2, 8, empty=(0, 1))
    assert len(a["w"]) == 0
    net = load(emr, a)
    gw, gx = check(emr, net, a, np.random.default_rng(3).uniform(-1, 1, (5, 2)), 3)
    assert gw.numel() == 0 and (gx == 0).all()


def test_hubs(emr):
    """One node that every node feeds and one that feeds every node, beside nodes without edges."""
    n_in, n_out, m = 2, 1, 700
    n = n_in + n_out + m
    rng = np.random.default_rng(0)
    src = [np.arange(n)] + [np.array([n_in + n_out])] * (m - 100) + [np.zeros(0, int)] * 100
    deg = [0] * n_in + [len(s) for s in src]
    a = {"subs": substrate(n_in, n_out), "is_in": np.array([True] * n_in + [False] * n_out),
         "node_offset": np.array([0, n]), "in_offset": np.concatenate([[0], np.cumsum(deg)]),
         "src": np.concatenate(src), "w": (rng.standard_normal(sum(deg)) * 0.2).astype(np.float32)}
    net = load(emr, a)
    check(emr, net, a, rng.uniform(-1, 1, (18, n_in)), 5)


def test_codes_at_their_ends(emr):
    """States of 0 and 255 (no slope) and all between."""
    a = random_nets(6, [50], 2, 2, 10)
    net = load(emr, a)
    x = np.random.default_rng(3).uniform(-1, 1, (9, 2))
    nodes = int(a["node_offset"][-1])
    codes = np.random.default_rng(4).choice([0, 1, 127, 128, 254, 255], (2, nodes, 9)).astype(np.uint8)
    codes[:, a["is_in"].nonzero()[0]] = 0
    check(emr, net, a, x, 3, codes=codes)
    gw, _ = check(emr, net, a, x, 3, codes=np.zeros_like(codes))
    inner = ~a["is_in"][np.minimum(a["src"], 3)] | (a["src"] > 3)
    assert (gw.cpu().numpy()[inner] == 0).all()


def test_gradient_against_differences(emr):
    """Central differences of the float64 activation's loss (h = 1e-5) against the kernel's gradient; the
    states' rounding to 8 bits moves a term of the gradient by at most 2 / 510 a step, relative to the
    terms' sizes."""
    a = random_nets(7, [6, 11], 3, 2, 5)
    net = load(emr, a)
    x = np.random.default_rng(5).uniform(-1, 1, (7, 3)).astype(np.float32).astype(np.float64)
    steps = 3
    rng = np.random.default_rng(6)
    grad_out = rng.standard_normal((2, 7, 2)).astype(np.float32)
    xd = torch.tensor(x, dtype=torch.float32, device="cuda")
    out, kept = net.activate_keep(xd, steps)
    gw, _ = net.activate_backward(xd, steps, out, kept, torch.tensor(grad_out, device="cuda"))

    def loss(w):
        s = forward64(dict(a, w=w), x, steps)[-1]
        return (s[output_nodes(a)].transpose(0, 2, 1) * grad_out).sum()

    c = np.rint(kept.values().double().cpu().numpy() * 255)
    _, _, aw, _ = backward64(a, x, steps, out.cpu().numpy(), c, grad_out)
    w = a["w"].astype(np.float64)
    # sizes of the terms at the steepest slope (1 / 4) instead of the codes' own
    _, _, bound, _ = backward64(a, x, steps, np.full_like(out.cpu().numpy(), 0.5),
                                np.full_like(c, 127.5), grad_out)
    for e in range(len(w)):
        d = np.zeros_like(w)
        d[e] = 1e-5
        want = (loss(w + d) - loss(w - d)) / 2e-5
        assert abs(want - float(gw[e])) <= steps * 2 / 510 * 4 * (bound[e] + aw[e]) + 1e-6


def test_built_networks_and_repeats(emr):
    """Networks of a population, with hidden nodes among themselves; the same bits on every call, and after
    the weights were set to others and back."""
    genomes = W.population(3, 30, 20, 60)
    subs = W.tabular_sources(5)
    pop = emr.emr_pack_population(genomes)
    net = emr.emr_build_networks(pop, subs, 5, 0.02, 15, 0.1, 1)
    a = from_handle(emr, net, subs)
    x = np.random.default_rng(5).uniform(-1, 1, (25, 5))
    gw, gx = check(emr, net, a, x, 3)
    assert (gw != 0).any()
    w = torch.tensor(a["w"], device="cuda")
    net.set_weights(w * 0.5)
    other, _ = check(emr, net, dict(a, w=a["w"] * np.float32(0.5)), x, 3)
    assert not torch.equal(other, gw)
    net.set_weights(w)
    np.testing.assert_array_equal(net.weights(), a["w"])
    again, gx2 = check(emr, net, a, x, 3)
    assert torch.equal(again, gw) and torch.equal(gx2, gx)
    copy = emr.emr_load_networks(subs, a["node_offset"], a["in_offset"], a["src"], a["w"])
    same, _ = check(emr, copy, a, x, 3)
    assert torch.equal(same, gw)


def test_streams_and_graph(emr):
    a = random_nets(8, [20, 90, 1500], 3, 2, 9)
    net = load(emr, a)
    xs = [torch.rand((10, 3), device="cuda") for _ in range(3)]
    g = torch.randn((3, 10, 2), device="cuda")
    want = []
    for x in xs:
        out, kept = net.activate_keep(x, 4)
        want.append((out, net.activate_backward(x, 4, out, kept, g, grad_inputs=True)))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, kept = net.activate_keep(xs[1], 4, stream=s)
    got = net.activate_backward(xs[1], 4, out, kept, g, grad_inputs=True, stream=s)
    s.synchronize()
    assert torch.equal(out, want[1][0]) and all(torch.equal(p, q) for p, q in zip(got, want[1][1]))
    still = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out, kept = net.activate_keep(still, 4)
        got = net.activate_backward(still, 4, out, kept, g, grad_inputs=True)
    for k in (0, 1, 2, 1):
        still.copy_(xs[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k][0])
        assert all(torch.equal(p, q) for p, q in zip(got, want[k][1]))
        eager, _ = net.activate_keep(xs[k], 4)
        assert torch.equal(eager, out)


def test_one_step_keeps_nothing(emr):
    a = random_nets(3, [7, 20], 2, 2, 6)
    net = load(emr, a)
    nodes = int(a["node_offset"][-1])
    x = torch.rand((5, 2), device="cuda")
    out, kept = net.activate_keep(x, 1)
    none = emr.kept_from_codes(torch.zeros((0, nodes, 5), dtype=torch.uint8, device="cuda"))
    assert kept.codes.shape == none.codes.shape and kept.values().shape == (0, nodes, 5)
    g = torch.randn_like(out)
    one, _ = net.activate_backward(x, 1, out, kept, g)
    two, _ = net.activate_backward(x, 1, out, none, g)
    assert torch.equal(one, two)


@pytest.mark.parametrize("patterns", [1, 4, 7, 8, 13, 16, 40, 100, 1000])
def test_kept_values(emr, patterns):
    """Codes to numbers of each type and back: what torch makes of them, to the bit."""
    g = torch.Generator(device="cuda").manual_seed(patterns)
    codes = torch.randint(0, 256, (2, 37, patterns), generator=g, device="cuda").to(torch.uint8)
    kept = emr.kept_from_codes(codes)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got = kept.values(dtype)
        want = (codes.float() * (1.0 / 255.0)).to(dtype)
        assert got.shape == codes.shape and torch.equal(got, want)
    with pytest.raises(ValueError):
        kept.values(torch.float64)


def test_refusals(emr):
    a = random_nets(9, [5, 8], 3, 2, 4)
    net = load(emr, a)
    x = torch.zeros((6, 3), device="cuda")
    out, kept = net.activate_keep(x, 3)
    with pytest.raises(ValueError):
        net.activate_keep(torch.zeros((6, 4), device="cuda"), 3)
    with pytest.raises(ValueError):
        net.activate_backward(x, 4, out, kept, out)  # states of another number of steps
    with pytest.raises(ValueError):
        net.activate_backward(x, 3, out, kept, out[:, :5])
    for bad in ((0, 3), (1 << 17, 3), (6, -1), (6, 1 << 21)):
        n = emr.C.c_int64()
        assert emr.lib().emr_kept_bytes(net.handle, *bad, emr.C.byref(n)) == emr.EMR_E_INVAL
    st = emr.lib().emr_activate_keep(net.handle, x.data_ptr(), 6, 3, out.data_ptr(), kept.codes.data_ptr(),
                                     kept.codes.numel() - 1, None)
    assert st == emr.EMR_E_CAPACITY
    st = emr.lib().emr_activate_keep(net.handle, x.data_ptr(), 6, 3, out.data_ptr(),
                                     kept.codes.data_ptr() + 4, 1 << 30, None)
    assert st == emr.EMR_E_INVAL
    with pytest.raises(ValueError):
        net.set_weights(torch.zeros(3, device="cuda"))
    good = (a["subs"], a["node_offset"], a["in_offset"], a["src"], a["w"])
    for k, v in ((1, a["node_offset"] + 1), (2, a["in_offset"][::-1].copy()), (3, a["src"] + 8)):
        bad = list(good)
        bad[k] = v
        with pytest.raises((emr.EmrError, ValueError)):
            emr.emr_load_networks(*bad)
    into_input = a["in_offset"].copy()
    into_input[1:4] = into_input[4]
    with pytest.raises(emr.EmrError) as e:
        emr.emr_load_networks(a["subs"], a["node_offset"], into_input, a["src"], a["w"])
    assert e.value.status == emr.EMR_E_INVAL


def test_graph_beside_other_calls(emr):
    """A captured call's replays give the same bits after calls on fewer and on more patterns, on more than 64
    numbers of them, on other handles; a call under capture that would lay out or allocate is refused, and
    the capture goes on."""
    a = random_nets(11, [900] + [60] * 40, 2, 1, 60)
    a = dict(a, w=a["w"] * np.float32(0.5))
    net, fresh = load(emr, a), load(emr, a)
    x = torch.rand((96, 2), device="cuda")
    g = torch.randn((41, 96, 1), device="cuda")
    want_out, kept = net.activate_keep(x, 3)
    want, _ = net.activate_backward(x, 3, want_out, kept, g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(emr.EmrError) as e:
            fresh.activate_keep(x, 3)
        assert e.value.status == emr.EMR_E_DEVICE
        with pytest.raises(emr.EmrError):
            net.activate_keep(x[:95], 3)
        out, kept = net.activate_keep(x, 3)
        got, _ = net.activate_backward(x, 3, out, kept, g)

    def others():
        for handle in (net, fresh):
            for patterns in [64, 700] + list(range(1, 70)):
                y = torch.rand((patterns, 2), device="cuda")
                o, k = handle.activate_keep(y, 2)
                handle.activate_backward(y, 2, o, k, torch.ones_like(o))

    for _ in range(2):
        out.zero_()
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_out) and torch.equal(got, want)
        others()
        torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want_out) and torch.equal(got, want)


def test_weights_set_by_a_graph(emr):
    """A graph that sets the weights, captured before and after the handle's first learning call: its replays
    count in the learning calls after them, captured ones too."""
    a = random_nets(12, [5, 40, 300], 3, 2, 9)
    x = torch.rand((9, 3), device="cuda")
    g = torch.randn((3, 9, 2), device="cuda")
    ws = [torch.tensor(a["w"] * np.float32(f), device="cuda") for f in (1.0, 0.5, -0.25)]
    want = []
    for w in ws:
        net = load(emr, dict(a, w=w.cpu().numpy()))
        out, kept = net.activate_keep(x, 3)
        want.append((out, net.activate_backward(x, 3, out, kept, g)[0]))
    for laid in (False, True):
        net = load(emr, a)
        if laid:
            net.activate_keep(x, 3)
        w = ws[0].clone()
        sets, learns = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(sets):
            net.set_weights(w)
        out, kept = net.activate_keep(x, 3)
        net.activate_backward(x, 3, out, kept, g)
        torch.cuda.synchronize()
        with torch.cuda.graph(learns):
            out_g, kept_g = net.activate_keep(x, 3)
            grad_g, _ = net.activate_backward(x, 3, out_g, kept_g, g)
        for k in (1, 2, 0, 1):
            w.copy_(ws[k])
            sets.replay()
            out, kept = net.activate_keep(x, 3)
            grad, _ = net.activate_backward(x, 3, out, kept, g)
            torch.cuda.synchronize()
            assert torch.equal(out, want[k][0]) and torch.equal(grad, want[k][1])
            learns.replay()
            torch.cuda.synchronize()
            assert torch.equal(out_g, want[k][0]) and torch.equal(grad_g, want[k][1])


def test_more_genomes_than_a_launch_takes(emr):
    """2^23 + 3 genomes of one edge, beyond what workgroups of one launch cover: their layouts, activation and
    gradients (sigmoid(w x), whatever the steps)."""
    G = (1 << 23) + 3
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("not enough free device memory")
    w = np.linspace(-2, 2, G).astype(np.float32)
    net = emr.emr_load_networks(substrate(1, 1), 2 * np.arange(G + 1), np.arange(2 * G + 1) // 2, 2 * np.arange(G), w)
    x = torch.tensor([[0.5], [-1.0]], device="cuda")
    out, kept = net.activate_keep(x, 2)
    want = torch.sigmoid(torch.tensor(w, device="cuda").double()[:, None, None] * x.double())
    # (the product's rounding, times the slope of at most 1 / 4, and the sigmoid's few of its own)
    assert (out.double() - want).abs().max() < 2.0 ** -21
    grad, _ = net.activate_backward(x, 2, out, kept, torch.ones_like(out))
    want = (want * (1 - want) * x.double()).sum((1, 2))
    assert (grad.double() - want).abs().max() < 2.0 ** -20


def test_many_patterns_of_large_genomes(emr):
    """More items than their sums' memory leaves room for (40 genomes of 4000 hidden nodes, 6000 patterns): the
    gradients of the first and the last genome against 64 bits."""
    G, m, deg, P, steps = 40, 4000, 60, 6000, 3
    n = m + 3
    rng = np.random.default_rng(0)
    d = np.array([0, 0, m] + [deg] * m)
    src = [np.concatenate([g * n + 3 + np.arange(m), g * n + np.sort(rng.integers(0, n, (m, deg)), axis=1).ravel()])
           for g in range(G)]
    a = {"subs": substrate(2, 1), "node_offset": n * np.arange(G + 1),
         "in_offset": np.concatenate([[0], np.cumsum(np.tile(d, G))]), "src": np.concatenate(src),
         "w": (rng.standard_normal(G * d.sum()) / 8).astype(np.float32)}
    net = load(emr, a)
    x = torch.rand((P, 2), device="cuda") * 2 - 1
    out, kept = net.activate_keep(x, steps)
    grad_out = torch.randn((G, P, 1), device="cuda") / P
    gw, gx = net.activate_backward(x, steps, out, kept, grad_out, grad_inputs=True)
    again, _ = net.activate_backward(x, steps, out, kept, grad_out)
    assert torch.equal(gw, again)
    e = int(d.sum())
    eps = unit(steps, max(P, m))
    to = torch.tensor(np.repeat(np.arange(n), d), device="cuda")
    for g in (0, G - 1):
        own = torch.tensor(src[g] - g * n, device="cuda")
        w = torch.zeros((n, n), dtype=torch.float64, device="cuda")
        w.index_put_((to, own), torch.tensor(a["w"][g * e:(g + 1) * e], device="cuda").double(), accumulate=True)
        # (the sizes of an edge's terms: of each of several edges between the same two nodes apart)
        size = torch.zeros_like(w).index_put_((to, own), torch.tensor(np.abs(a["w"][g * e:(g + 1) * e]),
                                                                     device="cuda").double(), accumulate=True)
        codes = kept.values()[:, g * n:(g + 1) * n].double()
        z = torch.zeros((n, P), dtype=torch.float64, device="cuda")
        o = out[g, :, 0].double()
        z[2] = grad_out[g, :, 0].double() * o * (1 - o)
        za, gm, ga = z.abs(), torch.zeros_like(w), torch.zeros_like(w)
        xs = torch.zeros((2, P), dtype=torch.float64, device="cuda")
        xa = xs.clone()
        for t in range(steps, 0, -1):
            s = codes[t - 2].clone() if t > 1 else torch.zeros_like(z)
            s[:2] = x.double().t()
            gm += z @ s.t().contiguous()
            ga += za @ s.abs().t().contiguous()
            back, size_back = w.t().contiguous() @ z, size.t().contiguous() @ za
            xs += back[:2]
            xa += size_back[:2]
            z, za = back * s * (1 - s), size_back * s * (1 - s)
            z[:2], za[:2] = 0, 0
        got = gw[g * e:(g + 1) * e].double()
        assert ((got - gm[to, own]).abs() <= eps * ga[to, own] + 1e-30).all()
        assert ((gx[g].double().t() - xs).abs() <= eps * xa + 1e-30).all()


@pytest.mark.parametrize("hidden", [[10300], [40, 10300, 0], [10236], [10237]])
def test_genomes_larger_than_any_layout(emr, hidden):
    """Genomes of more than 10239 nodes (and around that), alone and beside small ones: no layout, a launch for
    each step."""
    a = random_nets(sum(hidden), hidden, 2, 1, 6, mixed=True)
    net = load(emr, a)
    rng = np.random.default_rng(4)
    for patterns, steps in ((2, 1), (2, 3), (19, 3), (5, 4), (19, 0)):
        check(emr, net, a, rng.uniform(-1, 1, (patterns, 2)), steps)
    w = torch.tensor(a["w"], device="cuda")
    net.set_weights(w * -0.5)
    check(emr, net, dict(a, w=a["w"] * np.float32(-0.5)), rng.uniform(-1, 1, (9, 2)), 3)


def unrounded(a, x, steps, outputs_grad):
    """The weights' derivatives with no state rounded (float64), and a bound on what the states' rounding to 8
    bits and fp32 leave of it. A state's code errs by 1 / 510 and by what fp32 moved the state (a sum's chain of
    adds and the sigmoid's own, forward through the steps), an input not at all; s (1 - s) errs by no more than
    s does. So, backwards, with sizes |.| and errors e: e(gz s) <= e(gz) (|s| + e(s)) + |gz| e(s), and
    e(d s (1 - s)) <= e(d) (s (1 - s) + e(s)) + |d| e(s)."""
    G, P = len(a["node_offset"]) - 1, len(x)
    nodes = int(a["node_offset"][-1])
    held = np.concatenate([o + np.nonzero(a["is_in"])[0] for o in a["node_offset"][:-1]])
    degree = np.diff(a["in_offset"])
    dst, src, w = np.repeat(np.arange(nodes), degree), a["src"], a["w"].astype(np.float64)
    u = 2.0 ** -24

    def sums(at, of, weight, v):
        out = np.zeros((nodes, P))
        np.add.at(out, at, weight[:, None] * v[of])
        return out

    states = forward64(a, x, steps)
    fp32 = [np.zeros((nodes, P))]
    for t in range(steps):
        ez = sums(dst, src, np.abs(w), fp32[t]) + (degree[:, None] + 8) * u * sums(dst, src, np.abs(w), np.abs(states[t]))
        slope = states[t + 1] * (1 - states[t + 1])
        e = np.minimum(0.25, slope + 0.1 * ez) * ez + 4 * u  # (the sigmoid's second derivative is below 0.1)
        e[held] = 0
        fp32.append(e)
    err = [np.zeros((nodes, P))] + [e + 1 / 510 for e in fp32[1:]]
    for e in err:
        e[held] = 0
    at = output_nodes(a).reshape(-1)
    g = outputs_grad.astype(np.float64).transpose(0, 2, 1).reshape(-1, P)
    gz, ez = np.zeros((nodes, P)), np.zeros((nodes, P))
    o = states[steps][at]
    gz[at] = g * o * (1 - o)
    ez[at] = np.abs(g) * (fp32[steps][at] + 4 * u)
    gw, ew, size = np.zeros(len(src)), np.zeros(len(src)), np.zeros(len(src))
    za = np.abs(gz) + ez
    for t in range(steps, 0, -1):
        s, e = states[t - 1], err[t - 1]
        gw += (gz[dst] * s[src]).sum(1)
        ew += (ez[dst] * (np.abs(s) + e)[src] + np.abs(gz)[dst] * e[src]).sum(1)
        size += (za[dst] * (np.abs(s) + e)[src]).sum(1)
        d, ed, da = sums(src, dst, w, gz), sums(src, dst, np.abs(w), ez), sums(src, dst, np.abs(w), za)
        slope = np.abs(s * (1 - s))
        gz, ez, za = d * s * (1 - s), ed * (slope + e) + np.abs(d) * e, da * (slope + e)
        for v in (gz, ez, za):
            v[held] = 0
    terms = int(max(degree.max(), P, np.bincount(src).max()))
    return gw, ew + unit(steps, terms) * size


@pytest.mark.parametrize("inputs,types,iterations,steps", [(5, 15, 1, 3), (2, 1, 0, 2), (8, 15, 1, 5)])
def test_gradient_against_unrounded_states(emr, inputs, types, iterations, steps):
    """On discovered networks, in-degrees from none to hundreds."""
    subs = W.tabular_sources(inputs)
    pop = emr.emr_pack_population(W.population(3, 30, 20, 60))
    net = emr.emr_build_networks(pop, subs, 5, 0.02, types, 0.1, iterations)
    a = from_handle(emr, net, subs)
    assert len(a["w"]) > 1000
    rng = np.random.default_rng(1)
    x = rng.uniform(-1, 1, (21, int(a["is_in"].sum()))).astype(np.float32)
    grad_out = rng.standard_normal((30, 21, int((~a["is_in"]).sum()))).astype(np.float32)
    xd = torch.tensor(x, device="cuda")
    out, kept = net.activate_keep(xd, steps)
    gw, _ = net.activate_backward(xd, steps, out, kept, torch.tensor(grad_out, device="cuda"))
    want, bound = unrounded(a, x.astype(np.float64), steps, grad_out)
    assert np.abs(want).max() > 0
    assert (np.abs(gw.cpu().numpy() - want) <= bound + 1e-30).all()
