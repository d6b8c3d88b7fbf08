"""Example: fits a synthesis net to an image and decodes the image with it.

The net that the decoder runs for every pixel (Sec. 3.1: bilinear features of the
latent pyramid, an MLP, RGB) is trained here outside the decoder, on the GPU:

    forward    pic.linear          every layer, keeping what the gradient needs
    backward   pic.linear_backward into slices of one gradient buffer
    clipping   pic.GradClip        over the slices, in place

The parameters are one buffer in the layout of the decoder's weight blob, so the
trained net goes to pic.Decoder as it is.  The image to fit is the decode of
random weights of the same net ("teacher"), so that a fit exists.

With --images N, N nets are trained at once on an image each, and decoded as a batch:

    forward    pic.grouped_linear           every layer of all nets, rows sorted by image
    backward   pic.grouped_linear_backward  into slices of one gradient buffer
    clipping   pic.GradClip                 over all of it
    update     pic.Orthogonalizer           of the hidden layers' momenta; Adam for the rest

Run:  python -m paper_2609_09020_gb300.fit_net [--steps 400] [--net 7-64-64-3] [--size 192x256] [--dtype fp32] [--images 1]
"""
from __future__ import annotations

import argparse
import math

import numpy as np
import torch

from . import pic
from . import workloads as wk


def features(latents, steps, H, W, L, C):
    """[H * W][L * C] features: every level dequantised and upsampled to H x W
    (bilinear, half-pixel centres), as the decoder does it."""
    out, off = [], 0
    for level in range(L):
        h, w = -(-H >> level), -(-W >> level)
        q = latents[off:off + C * h * w].view(1, C, h, w).float() * steps[level]
        out.append(torch.nn.functional.interpolate(q, size=(H, W), mode="bilinear", align_corners=False)[0])
        off += C * h * w
    return torch.cat(out).reshape(L * C, H * W).t().contiguous()


class Net:
    """An MLP over one flat parameter buffer, blob layout (W_k, b_k, ...), and a
    gradient buffer of the same layout."""

    def __init__(self, dims, act, dtype, seed=0):
        self.dims, self.act = dims, act
        count = sum(n * (k + 1) for k, n in zip(dims, dims[1:]))
        self.master = torch.empty(count, device="cuda")  # fp32, what the optimiser changes
        self.params = self.master if dtype == torch.float32 else torch.empty(count, dtype=dtype, device="cuda")
        self.grads = torch.zeros_like(self.params)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for w, b in self.layers(self.master):
            w.normal_(0.0, math.sqrt(2.0 / w.shape[1]), generator=gen)
            b.zero_()
        self.params.copy_(self.master)

    def layers(self, buffer):
        out, off = [], 0
        for k, n in zip(self.dims, self.dims[1:]):
            out.append((buffer[off:off + n * k].view(n, k), buffer[off + n * k:off + n * (k + 1)]))
            off += n * (k + 1)
        return out

    def forward(self, x):
        """The output, and (input, pre-activation, activation) of every layer."""
        kept, layers = [], self.layers(self.params)
        for i, (w, b) in enumerate(layers):
            act = self.act if i + 1 < len(layers) else "none"
            y, z = pic.linear(x, w, b, act=act, save_pre=True)
            kept.append((x, z, act))
            x = y
        return x, kept

    def backward(self, dy, kept):
        """Fills the gradient buffer."""
        todo = list(zip(self.layers(self.params), self.layers(self.grads), kept))
        for i, ((w, _), (gw, gb), (x, z, act)) in reversed(list(enumerate(todo))):
            need = ("x", "weight", "bias") if i else ("weight", "bias")
            dy, _, _ = pic.linear_backward(dy, x, w, act=act, pre=z, need=need, dweight=gw, dbias=gb)


def fit(net, x, target, steps, lr=3e-3, max_norm=1.0, report=None):
    """Adam on the mean squared error; returns the losses."""
    clip = pic.GradClip([g for layer in net.layers(net.grads) for g in layer])
    m, v = torch.zeros_like(net.master), torch.zeros_like(net.master)
    # fp16 gradients of a mean are small: scale the loss, and the clipping with it
    scale = 1.0 if net.params.dtype == torch.float32 else 1024.0
    losses = []
    for step in range(1, steps + 1):
        y, kept = net.forward(x)
        diff = y.float() - target
        losses.append(diff.square().mean())
        net.backward((diff * (2.0 * scale / diff.numel())).to(y.dtype), kept)
        norm = clip.clip(max_norm * scale)
        g = net.grads.float() / scale
        m.lerp_(g, 0.1)
        v.lerp_(g * g, 0.01)
        rate = lr * min(1.0, 2.0 * (1.0 - step / (steps + 1)))
        net.master -= rate * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8)
        if net.params is not net.master:
            net.params.copy_(net.master)
        if report and (step == 1 or step % 100 == 0 or step == steps):
            report(f"step {step:5d}  loss {float(losses[-1]):.3e}  gradient norm {float(norm) / scale:.3e}")
    pic.linear_check()
    clip.check()
    clip.close()
    return [float(l) for l in losses]


class Nets:
    """`images` MLPs of one shape: parameters and gradients [images, count], each row a
    net's in blob layout."""

    def __init__(self, dims, act, dtype, images, seed=0):
        self.dims, self.act = dims, act
        nets = [Net(dims, act, dtype, seed + i) for i in range(images)]
        self.master = torch.stack([n.master for n in nets])
        self.params = self.master if dtype == torch.float32 else self.master.to(dtype)
        self.grads = torch.zeros_like(self.params)

    def layers(self, buffer):
        """(weights [images, out, in], biases [images, out]) of every layer: views of the buffer."""
        out, off = [], 0
        for k, n in zip(self.dims, self.dims[1:]):
            out.append((buffer[:, off:off + n * k].unflatten(1, (n, k)), buffer[:, off + n * k:off + n * (k + 1)]))
            off += n * (k + 1)
        return out

    def forward(self, x, offsets):
        """The output for rows sorted by image, and (input, pre-activation, activation) of every layer."""
        kept, layers = [], self.layers(self.params)
        for i, (w, b) in enumerate(layers):
            act = self.act if i + 1 < len(layers) else "none"
            y, z = pic.grouped_linear(x, w, offsets, b, act=act, save_pre=True)
            kept.append((x, z, act))
            x = y
        return x, kept

    def backward(self, dy, kept, offsets):
        """Fills the gradient buffer."""
        todo = list(zip(self.layers(self.params), self.layers(self.grads), kept))
        for i, ((w, _), (gw, gb), (x, z, act)) in reversed(list(enumerate(todo))):
            need = ("x", "weight", "bias") if i else ("weight", "bias")
            dy, _, _ = pic.grouped_linear_backward(dy, x, w, offsets, act=act, pre=z, need=need, dweight=gw, dbias=gb)


def fit_many(nets, x, target, offsets, steps, lr=3e-3, max_norm=1.0, report=None):
    """The nets' images at once; returns the mean squared errors [steps, images].  The weights
    between hidden layers take orthogonalised momenta, the others and the biases Adam."""
    images = nets.master.shape[0]
    clip = pic.GradClip([nets.grads])
    momentum, update = torch.zeros_like(nets.master), torch.zeros_like(nets.master)
    hidden = range(1, len(nets.dims) - 2)  # of layers
    w_of = lambda buffer: [nets.layers(buffer)[i][0] for i in hidden]
    orth = pic.Orthogonalizer(w_of(momentum), out=w_of(update))
    m, v = torch.zeros_like(nets.master), torch.zeros_like(nets.master)
    scale = 1.0 if nets.params.dtype == torch.float32 else 1024.0
    owner = torch.repeat_interleave(torch.arange(images, device="cuda"), torch.diff(offsets))
    rows = torch.diff(offsets).float() * target.shape[1]
    losses = []
    for step in range(1, steps + 1):
        y, kept = nets.forward(x, offsets)
        diff = y.float() - target
        losses.append(torch.zeros(images, device="cuda").index_add_(0, owner, diff.square().sum(1)) / rows)
        nets.backward((diff * (2.0 * scale / rows)[owner][:, None]).to(y.dtype), kept, offsets)
        clip.clip(max_norm * scale * images ** 0.5)
        g = nets.grads.float() / scale
        m.lerp_(g, 0.1)
        v.lerp_(g * g, 0.01)
        rate = lr * min(1.0, 2.0 * (1.0 - step / (steps + 1)))
        momentum.mul_(0.95).add_(g)
        adam = (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8)
        orth.orthogonalize()
        for a, u in zip(w_of(adam), w_of(update)):
            a.copy_(u)
        nets.master -= rate * adam
        if nets.params is not nets.master:
            nets.params.copy_(nets.master)
        if report and (step == 1 or step % 100 == 0 or step == steps):
            report(f"step {step:5d}  losses {float(losses[-1].min()):.3e} to {float(losses[-1].max()):.3e}")
    pic.grouped_linear_check()
    clip.check()
    clip.close()
    orth.check()
    orth.close()
    return torch.stack(losses)


def problems(dims, act, H, W, L, C, images, seed=0):
    """Of several images: latents [images, n], steps [images, L], and all their features, teachers' RGB and
    the images' first rows."""
    parts = [problem(dims, act, H, W, L, C, seed + i) for i in range(images)]
    offsets = torch.arange(images + 1, dtype=torch.int64, device="cuda") * (H * W)
    return (torch.stack([p[0].view(-1) for p in parts]), torch.stack([p[1].view(-1) for p in parts]),
            torch.cat([p[2] for p in parts]), torch.cat([p[3] for p in parts]), offsets)


def decode_many(nets, latents, steps, H, W, L, C):
    """RGB [images * H * W][3] of the trained nets, by the decoder in one batch."""
    images = latents.shape[0]
    dec = pic.Decoder(L, C, nets.dims, nets.act, "fp32", max_H=H, max_W=W, max_batch=images)
    rgb = torch.empty((images, 3, H, W), device="cuda")
    dec.decode_batch(latents, steps, nets.params.float(), H, W, rgb)
    dec.check()
    dec.close()
    return rgb.view(images, 3, H * W).transpose(1, 2).reshape(-1, 3)


def problem(dims, act, H, W, L, C, seed=0):
    """Latents (int32), steps, features and the teacher's RGB [H * W][3] of one image."""
    wl = wk.custom("fit", H=H, W=W, L=L, C=C, dims=dims, act=act, seed=seed)
    inputs = wk.make_inputs(wl)
    latents, steps = torch.from_numpy(inputs.latents).cuda(), torch.from_numpy(inputs.steps).cuda()
    dec = pic.Decoder(L, C, dims, act, "fp32", max_H=H, max_W=W)
    rgb = torch.empty((1, 3, H, W), device="cuda")
    dec.decode(latents, steps, torch.from_numpy(inputs.weights_for("fp32")).cuda(), H, W, rgb)
    dec.check()
    dec.close()
    x = features(latents.view(-1), steps.view(-1), H, W, L, C)
    return latents, steps, x, rgb[0].reshape(3, H * W).t().contiguous()


def decode(net, latents, steps, H, W, L, C):
    """RGB [H * W][3] of the trained net, by the decoder."""
    dec = pic.Decoder(L, C, net.dims, net.act, "fp32", max_H=H, max_W=W)
    rgb = torch.empty((1, 3, H, W), device="cuda")
    # the decoder reads weights on a 16-byte boundary: the blob is a buffer of its own
    dec.decode(latents, steps, net.params.float(), H, W, rgb)
    dec.check()
    dec.close()
    return rgb[0].reshape(3, H * W).t()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--net", default="7-64-64-3")
    ap.add_argument("--act", default="relu", choices=["relu", "gelu"])
    ap.add_argument("--size", default="192x256")
    ap.add_argument("--dtype", default="fp32", choices=["fp32", "fp16", "bf16"])
    ap.add_argument("--images", type=int, default=1)
    a = ap.parse_args(argv)
    dims = tuple(int(d) for d in a.net.split("-"))
    H, W = (int(d) for d in a.size.split("x"))
    L, C = dims[0], 1
    dtype = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[a.dtype]
    if a.images > 1:
        latents, steps, x, target, offsets = problems(dims, a.act, H, W, L, C, a.images)
        nets = Nets(dims, a.act, dtype, a.images, seed=1)
        fit_many(nets, x.to(dtype), target, offsets, a.steps, report=print)
        mse = (decode_many(nets, latents, steps, H, W, L, C) - target).square().view(a.images, -1).mean(1).clamp(min=1e-20)
        psnr = -10 * torch.log10(mse)
        print(f"decoded with the trained nets: PSNR {float(psnr.min()):.1f} to {float(psnr.max()):.1f} dB against the images")
        return
    latents, steps, x, target = problem(dims, a.act, H, W, L, C)
    net = Net(dims, a.act, dtype, seed=1)
    fit(net, x.to(dtype), target, a.steps, report=print)
    mse = float((decode(net, latents, steps, H, W, L, C) - target).square().mean())
    print(f"decoded with the trained net: PSNR {-10 * np.log10(max(mse, 1e-20)):.1f} dB against the image")


if __name__ == "__main__":
    main()
