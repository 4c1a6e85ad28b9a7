"""What the operators around the products launch, at the edges of their rules (host code: nothing is launched)."""
import math
import random

import pytest

from dispatch_train import dispatch

F32, BF16 = 0, 1


@pytest.mark.parametrize("B,P,C,G,dtype,off", [(65535, 1, 33800, 65, BF16, 0), (65535, 1, 60000, 100, BF16, 0), (65535, 10, 65536, 128, BF16, 1),
                                               (65535, 323, 2964, 78, BF16, 1), (16926, 9, 65536, 256, F32, 1), (65468, 1, 65500, 100, BF16, 0)])
def test_normalisations_of_many_groups_are_launched(B, P, C, G, dtype, off):
    """As many images and groups as are taken: more threads than 32 bits count would be an image's channels in
    registers each."""
    for call in dispatch([(kind, B, P, C, G, dtype, off, act) for kind in ("norm_fwd", "norm_bwd") for act in range(3)]):
        assert call.rc == 0, call


@pytest.mark.parametrize("M,K,N", [(4194240, 16536, 3), (11, 2097112, 32663), (4194145, 16637, 1), (1, 2097152, 33327)])
@pytest.mark.parametrize("off", [0, 1])
def test_operands_of_any_size_are_packed(M, K, N, off):
    """More features and rows, or classes, than a launch has threads for at eight rows and two columns each."""
    for call in dispatch([("xent_fwd", M, K, N, off, BF16, 1), ("xent_step", M, K, N, off, BF16, 1, 6)]):
        assert call.rc == 0, call


def _size(rng, lo, hi):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return rng.choice((lo, hi, hi - rng.randint(0, 99), max(lo, min(hi, round(v))), max(lo, min(hi, round(v)))))


@pytest.mark.parametrize("seed", range(4))
def test_what_the_memory_holds_is_launched(seed):
    """Sizes at random, up to the largest that are taken, of which tensors and workspace are at most 288 GB."""
    rng, calls, held = random.Random(seed), [], []
    while len(calls) < 2000:
        dtype, off = rng.randint(0, 1), rng.randint(0, 1)
        size = 2 if dtype else 4
        if rng.random() < 0.5:
            C = _size(rng, 100, 65536)
            G = rng.choice([d for d in (1, 2, 3, 4, 5, 8, 10, 16, 32, 50, 64, 100, 128, 256, 1024, C) if C % d == 0])
            images, P = _size(rng, 100, 65535), _size(rng, 100, (1 << 31) - 1) // 100
            if images * G > 1 << 23:
                continue
            calls.append((rng.choice(("norm_fwd", "norm_bwd")), images, P, C, G, dtype, off, rng.randint(0, 2)))
            held.append(2 * images * P * C * size)
        else:
            M, K, N = _size(rng, 100, 4194240) // rng.choice((1, 100)), _size(rng, 100, 1 << 21), _size(rng, 100, 4194240) // rng.choice((1, 100))
            need = rng.randint(1, 7)
            kind = rng.choice(("xent_fwd", "xent_bwd", "xent_step"))
            calls.append((kind, M, K, N, off, dtype, rng.randint(0, 2), need))
            grads = 0 if kind == "xent_fwd" else (need & 1) * M * K + (need >> 1 & 1) * K * N
            held.append((M * K + K * N + grads) * size)
    fit = 0
    for call, tensors, got in zip(calls, held, dispatch(calls)):
        if tensors + got.workspace <= 288e9:
            fit += 1
            assert got.rc == 0, (call, got)
    assert fit > 400


def test_normalisations_without_slices_hold_no_sums_of_slices():
    """A workspace is for what a call writes into it: with an image's channels in registers nothing forward, and the images'
    sums of their channels backward."""
    sizes = [(128, 1024, 64, 32, F32), (128, 16, 512, 32, F32), (65535, 1, 256, 8, BF16), (4096, 1, 8192, 64, F32), (1, 49, 96, 3, BF16)]
    for (images, P, C, G, dtype), fwd, bwd in zip(sizes, dispatch([("norm_fwd",) + s for s in sizes]), dispatch([("norm_bwd",) + s for s in sizes])):
        assert all("sums" not in k for k in fwd.kernels + bwd.kernels)
        assert 0 < fwd.workspace <= 256 and 0 < bwd.workspace <= 8 * images * C + 256, (fwd, bwd)


def _cdiv(a, b):
    return -(-a // b)


@pytest.mark.parametrize("M,K,N", [(777, 320, 10007), (512, 2048, 1000), (10000, 512, 1000), (1000000, 512, 1000), (200000, 32, 1024), (3000000, 8, 20),
                                   (40000, 32, 4321), (9001, 520, 6001)])
def test_backward_calls_keep_no_logits(M, K, N):
    """In fp32, where a step may keep them: a workspace of X and W in planes, dz of a piece in planes (128 MB, or 1024
    classes), sums over rows for dbias, and sums of parts.  A step's logits are 128 MB at most."""
    bwd, step = dispatch([("xent_bwd", M, K, N, 0, F32, 1, 7), ("xent_step", M, K, N, 0, F32, 1, 7)])
    assert bwd.rc == step.rc == 0 and not any("dz_kernel" in k for k in bwd.kernels)
    piece = min(N, max(1024, (128 << 20) // (6 * M) // 256 * 256))
    planes = 6 * (M * _cdiv(K, 32) * 32 + K * _cdiv(N, 32) * 32)
    dz, eights = 6 * M * _cdiv(piece, 256) * 256, 4 * _cdiv(M, 8 if piece == N and 4 * M * _cdiv(N, 256) * 256 <= 128 << 20 else 64) * piece
    parts = 4 * 64 * max(M * K if M * K <= 1 << 24 else 0, K * N)          # (few outputs come in parts)
    sums = 4 * M * K if piece < N or M * K <= 1 << 24 else 0
    assert bwd.workspace <= planes + dz + eights + parts + sums + 4096
    assert step.workspace - bwd.workspace <= (128 << 20) + 16 * M * _cdiv(N, 128)


def test_the_tests_of_values_reach_the_large_kernels():
    """Both tiles of either type, the launch that makes dz from logits that a step has kept, and dX over several pieces."""
    import torch
    from test_gpu_xent_edges import LARGE

    seen = set()
    for dtype, code in ((torch.float32, F32), (torch.bfloat16, BF16)):
        for size in LARGE[dtype]:
            for what in ("xent_step", "xent_bwd"):
                call = dispatch([(what, *size, 0, code, 1, 7)])[0]
                assert call.rc == 0 and not any("small" in k for k in call.kernels), call
                seen.update(call.kernels)
                if sum(k.startswith("xent_gradient_kernel") for k in call.kernels) > 2:
                    seen.add(f"pieces {code}")
    for planes, tiles in ((1, ("256, 256", "128, 128")), (3, ("256, 128", "128, 64"))):
        for tile in tiles:
            for grad in ("false", "true"):
                assert any(k.startswith(f"xent_logits_kernel<{grad}, {planes}, {tile}") for k in seen), (grad, planes, tile)
            for mode in (0, 1):
                assert any(k.startswith(f"xent_gradient_kernel<{planes}, {mode}, {tile}") for k in seen), (mode, planes, tile)
    assert "xent_dz_kernel" in seen and {"pieces 0", "pieces 1"} <= seen


@pytest.mark.parametrize("M,K,N,dtype", [(512, 512, 1000, F32), (8192, 64, 100, F32), (1, 256, 4000, BF16), (2048, 32, 700, BF16)])
def test_forward_calls_of_small_problems_hold_no_logits(M, K, N, dtype):
    """Only gradients read them: a forward call's workspace is the rows' pairs, eight bytes for each 32 classes, and two words a row."""
    fwd, bwd = dispatch([(what, M, K, N, 0, dtype, 1, 7) for what in ("xent_fwd", "xent_bwd")])
    assert fwd.rc == bwd.rc == 0 and any("small_logits" in k for k in fwd.kernels)
    assert fwd.workspace <= 8 * M * _cdiv(N, 32) + 8 * M + 768 and bwd.workspace >= 4 * M * N
