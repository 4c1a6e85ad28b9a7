"""Class incremental training of the CIFAR-width ResNet-18 on synthetic images: every matmul of the network quantized,
group normalisation between the layers, the growing classifier's loss and the clipping of the gradients by the
library.

    python -m paper_2310_03675_amd.train --tasks 2 --steps 20

Each task brings an equal share of the classes; the classifier's columns of later tasks are not in use until then.
Images are noise around a pattern of their class (no dataset is needed); seeds are fixed.
"""
import argparse
from typing import Iterator, List, Tuple

import torch

from .autograd import LayerConfig, clip_gradients
from .resnet import ResNet18


def batches(patterns: torch.Tensor, first: int, last: int, size: int, steps: int, seed: int) -> Iterator[Tuple[torch.Tensor, torch.Tensor]]:
    """Images of the classes [first, last): the class's pattern under noise."""
    g = torch.Generator(device=patterns.device).manual_seed(seed)
    for _ in range(steps):
        labels = torch.randint(first, last, (size,), device=patterns.device, generator=g)
        noise = torch.randn((size,) + tuple(patterns.shape[1:]), device=patterns.device, generator=g)
        yield patterns[labels] + 0.5 * noise, labels


def train(tasks: int = 2, steps: int = 20, classes: int = 100, batch: int = 128, lr: float = 0.05, max_norm: float = 1.0,
          seed: int = 0, device: str = "cuda:0", report=print) -> List[Tuple[float, float]]:
    """-> (loss, gradient norm before clipping) of every step."""
    if tasks < 1 or classes % tasks:
        raise ValueError(f"{classes} classes are no whole tasks of {tasks}")
    torch.manual_seed(seed)
    patterns = torch.randn(classes, 3, 32, 32, device=device)
    net = ResNet18(classes, base=LayerConfig(seed=seed), device=device, norm="group", head="loss").train()
    opt = torch.optim.SGD(net.parameters(), lr=lr, momentum=0.9, weight_decay=5e-4)
    history = []
    for task in range(tasks):
        last = classes // tasks * (task + 1)
        net.head.classes = last
        for step, (images, labels) in enumerate(batches(patterns, last - classes // tasks, last, batch, steps, seed + task)):
            opt.zero_grad(set_to_none=True)
            loss = net(images, labels)
            loss.backward()
            norm = clip_gradients(net.parameters(), max_norm)
            opt.step()
            history.append((loss.detach(), norm))
            if report and (step + 1) % 10 == 0:
                report(f"task {task + 1}, step {step + 1}: loss {float(loss.detach()):.4f}, gradient norm {float(norm):.3f}")
    return [(float(a), float(b)) for a, b in history]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tasks", 2), ("steps", 20), ("classes", 100), ("batch", 128), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    for name, value in (("lr", 0.05), ("max-norm", 1.0)):
        ap.add_argument(f"--{name}", type=float, default=value)
    train(**vars(ap.parse_args()))


if __name__ == "__main__":
    main()
