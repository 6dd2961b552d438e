"""Dense operators before and behind a net's run, on one stream without a wait between them (each starts while the one before it ends), and beside
nets on other streams: everything has the results that it has alone."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2011_05630_b200 import binding as B, dense, networks as nw, synth
from paper_2011_05630_b200.runtime import Session
from tests.test_gpu_dense import Maker


def session(layers, tag, n, h, w, c, plan=None):
    sess = Session(layers, synth.layer_params(tag, layers), n, h, w, c)
    if plan is None:
        sess.set_plan()
    else:
        sess.set_plan(*plan)
    return sess, sess.upload(synth.network_input(tag, n, h, w, c))


def run(sess, x):
    """Enqueues a run; a copy of its output."""
    B.net_run(sess.net, x.data_ptr(), sess.out.data_ptr(), torch.cuda.current_stream().cuda_stream)
    return sess.out.clone()


NETS = {"group": (nw.two_layer_group, 1, 32, 32, 16, ([1], [4])), "layers": (nw.two_layer_group, 1, 32, 32, 16, None), "resnet18": (nw.resnet18, 2, 224, 224, 3, None),
        "mobilenet": (nw.mobilenet_v2, 1, 224, 224, 3, None)}


@pytest.mark.parametrize("m", [5, 300])
@pytest.mark.parametrize("name", list(NETS))
def test_in_a_row(name, m):
    make, n, h, w, c, plan = NETS[name]
    layers = make()
    sess, x0 = session(layers, "row-" + name, n, h, w, c, plan)
    mk = Maker(m, torch.float16)
    k = 48 if c == 3 else 64   # (values of the input in rows of k)
    tokens = x0.numel() // k
    w1 = (torch.eye(k, device="cuda") * 0.5).half() + mk.mat(k, k, 0.1 / k ** 0.5)
    width = sess.out.shape[-1]
    wg, wu, wd = mk.mat(704, width, width ** -0.5), mk.mat(704, width, width ** -0.5), mk.mat(width, 704, 704 ** -0.5)

    def once(wait):
        sync = torch.cuda.synchronize if wait else lambda: None
        a = dense.linear(x0.view(tokens, k), w1, act="silu")
        sync()
        f = run(sess, a)
        sync()
        f = f.view(-1, width)[:m]
        hh, g, u = dense.gated(f, wg, wu, save=True)
        sync()
        y = dense.linear(hh, wd, residual=f)
        sync()
        dh, dwd, _, _ = dense.linear_backward(y, hh, wd, bias=False)
        sync()
        return [a, f, hh, y, dh, dwd, *[t for t in dense.gated_backward(dh, f, wg, wu, g, u) if t is not None]]

    want = once(True)
    for _ in range(10):
        got = once(False)
    B.net_sync(sess.net, torch.cuda.current_stream().cuda_stream)
    dense.synchronize()
    assert all(bool(torch.isfinite(t).all()) for t in want)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    sess.close()


def test_side_by_side():
    """Two nets and dense operators of every kind, a stream each."""
    nets = [session(nw.resnet18(), "side-a", 2, 224, 224, 3), session(nw.mobilenet_v2(), "side-b", 1, 224, 224, 3)]
    mk = Maker(4, torch.bfloat16)
    work = []
    for m, k, n in ((3, 1024, 2816), (40, 2048, 1024), (300, 512, 1408), (2048, 512, 2048)):
        work.append((mk.mat(m, k), mk.mat(n, k, k ** -0.5), mk.mat(n, k, k ** -0.5), mk.mat(m, n)))

    def operators():
        out = []
        for x, w, wu, dy in work:
            h, g, u = dense.gated(x, w, wu, save=True)
            out += [h, *dense.linear_backward(dy, x, w)[:3], *dense.gated_backward(dy, x, w, wu, g, u, bias=True)]
        return out

    calls = [lambda: [run(*nets[0])], lambda: [run(*nets[1])], operators, operators]
    want = []
    for call in calls:
        want.append(call())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [None] * len(calls)
    for _ in range(8):
        for i, call in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                got[i] = call()
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            if i < 2:
                B.net_sync(nets[i][0].net, s.cuda_stream)
            dense.synchronize()
    for i in range(len(calls)):
        assert all(torch.equal(p, q) for p, q in zip(got[i], want[i])), i
    for sess, _ in nets:
        sess.close()
