"""A small network learns from a quantized teacher: what the distillation operators are for, run together.

    python -m paper_1903_12650_amd.distill_example [--steps 40] [--batch 40] [--classes 1000]

The teacher only answers: a fixed convolution, global average pooling and a wide classifier whose weights are quantized once
(quant_rows_i8) and multiplied in 8-bit integers (fc_i8_fwd); of its logits the largest are kept (topk_rows), which is also all that
a program would store of them.  The student is trained: convolution, batch norm + ReLU, pooling, classifier, the loss against the
teacher's logits and the labels (distill_fwd_bwd), the backward pass of all of it, and LARS on single-precision weights with a
bfloat16 copy.  Images are synthetic, labels the teacher's first choices."""
import argparse

import torch

import paper_1903_12650_amd as rn


class Teacher:
    def __init__(self, classes, channels=64, width=2048, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)
        self.conv = (rand(width, 3, 3, channels) * (2 / (9 * channels)) ** 0.5).bfloat16()
        # (pooled features are near their mean: a classifier that tells images apart has large weights)
        self.w, self.w_scale = rn.quant_rows_i8(rand(classes, width) * 0.6)
        self.bias = torch.zeros(classes, device="cuda")

    def entries(self, images, k, temperature):
        """The k largest logits of every image, their classes, and the log-sum-exp of the others at the temperature."""
        y = rn.conv_fwd(images, self.conv, 1, 1)
        features = rn.avgpool_fwd(torch.relu(y))
        return rn.topk_rows(rn.fc_i8_fwd(features, self.w, self.w_scale, self.bias), k, temperature)


class Student:
    def __init__(self, classes, channels=64, width=256, seed=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)
        # single-precision weights: convolution, batch norm's scale and centre, classifier and its bias; trained in this order
        self.master = [rand(width, 3, 3, channels) * (2 / (9 * channels)) ** 0.5, torch.ones(width, device="cuda"),
                       torch.zeros(width, device="cuda"), rand(classes, width) * width ** -0.5, torch.zeros(classes, device="cuda")]
        self.model = [w.bfloat16() for w in self.master]
        self.grads = [torch.empty_like(w) for w in self.master]
        velocity = [torch.zeros_like(w) for w in self.master]
        decay = [5e-5, 0.0, 0.0, 5e-5, 0.0]
        self.table = rn.LarsTable(self.master, self.grads, velocity, decay, [1, 0, 0, 1, 0], self.model)

    def step(self, images, entries, labels, temperature, alpha, label_smoothing, lr):
        values, indices, tail = entries
        conv, fc = self.model[0], self.model[3]
        gamma, beta, bias = self.master[1], self.master[2], self.master[4]
        n, h, w, _ = images.shape
        y = rn.conv_fwd(images, conv, 1, 1)
        z, mean, rstd = rn.bn_relu_fwd(y, gamma, beta)
        a = rn.avgpool_fwd(z)
        logits = rn.fc_fwd(a, fc, bias)
        # the gradient takes the logits' place
        loss, _, dlogits = rn.distill_fwd_bwd(logits, values, indices, tail, labels, temperature, alpha, label_smoothing, dlogits=logits)
        da, dfc, dbias = rn.fc_bwd(a, fc, dlogits)
        dy, _, dgamma, dbeta = rn.bn_relu_bwd(rn.avgpool_bwd(da, h, w), y, z, gamma, mean, rstd, beta=beta)
        dconv = rn.conv_wgrad(images, dy, conv.shape, 1, 1)
        for g, d in zip(self.grads, (dconv, dgamma, dbeta, dfc, dbias)):
            g.copy_(d)
        rn.lars_update(self.table, 0.001, 0.9, lr)
        return loss


def run(steps=40, batch=40, classes=1000, k=16, temperature=2.0, alpha=0.7, label_smoothing=0.1, lr=5.0, batches=4, seed=3):
    """Trains the student for some steps; returns the losses (a device tensor)."""
    teacher, student = Teacher(classes), Student(classes)
    g = torch.Generator(device="cuda").manual_seed(seed)
    images = [torch.randn((batch, 8, 8, 64), device="cuda", generator=g).bfloat16() for _ in range(batches)]
    entries = [teacher.entries(x, k, temperature) for x in images]
    losses = []
    for i in range(steps):
        x, e = images[i % batches], entries[i % batches]
        losses.append(student.step(x, e, e[1][:, 0].contiguous(), temperature, alpha, label_smoothing, lr))
    return torch.cat(losses)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--batch", type=int, default=40)
    ap.add_argument("--classes", type=int, default=1000)
    a = ap.parse_args()
    losses = run(a.steps, a.batch, a.classes).tolist()
    for i in range(0, a.steps, max(1, a.steps // 8)):
        print(f"step {i}: loss {losses[i]:.4f}")
    print(f"last: loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
