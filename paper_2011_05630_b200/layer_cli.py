"""Command line for one layer: builds a single convolution / depthwise / max-pool layer, or one fused inverted-residual
block, with the seeded synthetic tensors of the workloads, runs it a few times through the C ABI and prints which kernel
ran (handy under a profiler, or to try a shape before putting it into a network).

    python -m paper_2011_05630_b200.layer_cli N H W CIN COUT K [--as-chain] [--reps 3] [--stride 1]
                                              [--op conv|dwconv|maxpool] [--mbconv HID]
                                              [--then K:C,K:C,...] [--residual] [--group-kernel 0|1|2]
                                              [--op linear|gated [--act silu] [--dtype bf16] [--backward]]

--then appends dense stride-1 convolutions (kernel:channels) and runs all of them as ONE group; --residual adds the
group's input to its last layer; --group-kernel picks the hand-over (1 shared memory, 2 L2, 0 the library's choice).
--op dwconv runs a depthwise KxK layer (COUT = CIN), --op maxpool a KxK max-pool; --mbconv HID runs the fused
inverted-residual block CIN -> HID (1x1) -> depthwise 3x3 (--stride) -> COUT (1x1) as one group.
--op linear runs the dense operator act(x w^T + bias [+ residual]) on N*H*W tokens of CIN -> COUT values (K is not used), --op gated the gated
block's act(x wg^T) * (x wu^T), --backward their gradients, too; each prints its time on the device and the kernels that ran.
"""
from __future__ import annotations

import argparse


def dense_op(a):
    """One dense operator with seeded tensors: forwards, and backwards if asked for."""
    import torch
    from . import dense
    dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[a.dtype]
    act = a.act or ("silu" if a.op == "gated" else "none")
    gen = torch.Generator(device="cuda").manual_seed(0)
    mat = lambda rows, cols, scale=1.0: (torch.randn((rows, cols), generator=gen, device="cuda") * scale).to(dtype)
    m, k, n = a.n * a.h * a.w, a.cin, a.cout
    x, dy, w, wu = mat(m, k), mat(m, n), mat(n, k, k ** -0.5), mat(n, k, k ** -0.5)
    bias, res = torch.randn((n,), generator=gen, device="cuda") * 0.1, mat(m, n) if a.residual else None
    kept = dense.linear(x, w, bias, res, act=act, save=True) if a.op == "linear" else dense.gated(x, w, wu, act=act, save=True)
    calls = {"forward": (lambda: dense.linear(x, w, bias, res, act=act)) if a.op == "linear" else (lambda: dense.gated(x, w, wu, act=act))}
    if a.backward:
        calls["backward"] = ((lambda: dense.linear_backward(dy, x, w, kept[1], act=act, residual=a.residual)) if a.op == "linear"
                             else (lambda: dense.gated_backward(dy, x, w, wu, kept[1], kept[2], act=act)))
    for name, call in calls.items():
        ran, = dense.kernels(call)
        ends = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ends[0].record()
        for _ in range(a.reps):
            call()
        ends[1].record()
        dense.synchronize()
        print("%s %s, %d tokens of %d -> %d, %s, act %s: %.2f us a call, x %d" % (a.op, name, m, k, n, a.dtype, act, ends[0].elapsed_time(ends[1]) * 1e3 / a.reps, a.reps))
        print("  " + ran)


def main():
    ap = argparse.ArgumentParser()
    for name in ("n", "h", "w", "cin", "cout", "k"):
        ap.add_argument(name, type=int)
    ap.add_argument("--as-chain", action="store_true", help="use the fused-chain kernel for the single layer")
    ap.add_argument("--reps", type=int, default=3)
    ap.add_argument("--stride", type=int, default=1)
    ap.add_argument("--op", default="conv", choices=["conv", "dwconv", "maxpool", "linear", "gated"])
    ap.add_argument("--mbconv", type=int, default=0, help="hidden width of a fused inverted-residual block")
    ap.add_argument("--then", default="", help="more dense convolutions K:C,K:C,... fused with the first into one group")
    ap.add_argument("--residual", action="store_true", help="add the group's input to its last layer (channels must match)")
    ap.add_argument("--group-kernel", type=int, default=0, choices=[0, 1, 2])
    ap.add_argument("--act", default=None, choices=["none", "relu", "relu6", "gelu", "gelu_tanh", "silu"], help="of a dense operator")
    ap.add_argument("--dtype", default="f16", choices=["f16", "bf16"], help="of a dense operator's matrices")
    ap.add_argument("--backward", action="store_true", help="a dense operator's gradients, too")
    a = ap.parse_args()
    if a.op in ("linear", "gated"):
        return dense_op(a)
    from . import binding as B
    from .runtime import Session
    def mk(op, cin, cout, k, stride, src, act="relu", res=-2):
        return dict(op=op, act=act, cin=cin, cout=cout, kh=k, kw=k, stride=stride, pad=k // 2, groups=cin if op == "dwconv" else 1,
                    src=src, res_src=res, pool=0)
    if a.mbconv:
        res = -1 if (a.stride == 1 and a.cin == a.cout) else -2
        layers = [mk("conv", a.cin, a.mbconv, 1, 1, -1, "relu6"), mk("dwconv", a.mbconv, a.mbconv, 3, a.stride, 0, "relu6"),
                  mk("conv", a.mbconv, a.cout, 1, 1, 1, "none", res)]
    else:
        layers = [mk(a.op, a.cin, a.cin if a.op != "conv" else a.cout, a.k, a.stride, -1, "none" if a.op == "maxpool" else "relu")]
    for spec in [t for t in a.then.split(",") if t]:
        k, c = (int(v) for v in spec.split(":"))
        layers.append(mk("conv", layers[-1]["cout"], c, k, 1, len(layers) - 1))
    if a.residual:
        layers[-1]["res_src"] = -1
    from . import synth
    params = synth.layer_params("layer_cli", layers)
    x = synth.network_input("layer_cli", a.n, a.h, a.w, a.cin)
    sess = Session(layers, params, a.n, a.h, a.w, a.cin)
    xd = sess.upload(x)
    B.net_set_option(sess.net, B.OPT_CUDA_GRAPH, 0)
    B.net_set_option(sess.net, B.OPT_SINGLE_AS_CHAIN, 1 if a.as_chain else 0)
    B.net_set_option(sess.net, B.OPT_GROUP_KERNEL, a.group_kernel)
    sess.set_plan([len(layers) - 1], [B.device_sm_count()])
    for _ in range(a.reps):
        sess.run(xd)
    print("ran", sess.launches(), "x", a.reps)


if __name__ == "__main__":
    main()
