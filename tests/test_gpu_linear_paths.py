"""Every way that a linear layer's product can go, by an odd and an even size each: which kernel, which tiles, whether the sum is
taken in parts.  test_linear_paths_host.py asks that there is no other one, and that these sizes go where they say.

Bounds as in test_gpu_linear.py: with e = 2^-24 a float32 sum of k products is within (k + 8) 2 e of the sum of the products'
magnitudes, which covers what taking float32 apart leaves out; a bfloat16 result is rounded by 2^-8 at most."""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16}
KERNELS = ["few", "product", "lone", "product3", "raw3"]
PASSES = ["forward", "dx", "dw"]

# type, pass, kernel, rows of a tile, sum in parts, (rows, features in, features out)
PATHS = [
    ("f32", "forward", "few", 0, False, (4, 205, 65)),
    ("f32", "forward", "few", 0, False, (4, 256, 64)),
    ("f32", "forward", "product3", 128, False, (2595, 203, 2625)),
    ("f32", "forward", "product3", 128, False, (2752, 256, 2560)),
    ("f32", "forward", "product3", 128, True, (3105, 2299, 2627)),
    ("f32", "forward", "product3", 128, True, (2432, 2304, 3392)),
    ("f32", "forward", "raw3", 128, False, (461, 201, 327)),
    ("f32", "forward", "raw3", 128, False, (832, 256, 320)),
    ("f32", "forward", "raw3", 128, True, (18, 217, 67)),
    ("f32", "forward", "raw3", 128, True, (17, 256, 64)),
    ("f32", "dx", "product3", 128, False, (324, 463, 205)),
    ("f32", "dx", "product3", 128, False, (320, 832, 256)),
    ("f32", "dx", "product3", 128, True, (4, 65, 201)),
    ("f32", "dx", "product3", 128, True, (4, 64, 256)),
    ("f32", "dw", "product3", 128, False, (201, 331, 463)),
    ("f32", "dw", "product3", 128, False, (256, 320, 832)),
    ("f32", "dw", "product3", 128, True, (206, 65, 65)),
    ("f32", "dw", "product3", 128, True, (256, 64, 64)),
    ("bf16", "forward", "few", 0, False, (4, 205, 65)),
    ("bf16", "forward", "few", 0, False, (4, 256, 64)),
    ("bf16", "forward", "lone", 128, False, (66, 207, 69)),
    ("bf16", "forward", "lone", 128, False, (128, 256, 64)),
    ("bf16", "forward", "lone", 128, True, (67, 641, 71)),
    ("bf16", "forward", "lone", 128, True, (128, 704, 64)),
    ("bf16", "forward", "product", 32, False, (18, 217, 67)),
    ("bf16", "forward", "product", 32, False, (17, 256, 64)),
    ("bf16", "forward", "product", 32, True, (17, 463, 67)),
    ("bf16", "forward", "product", 32, True, (17, 512, 64)),
    ("bf16", "forward", "product", 64, False, (33, 207, 71)),
    ("bf16", "forward", "product", 64, False, (33, 256, 64)),
    ("bf16", "forward", "product", 64, True, (42, 459, 65)),
    ("bf16", "forward", "product", 64, True, (33, 512, 64)),
    ("bf16", "forward", "product", 128, False, (8707, 201, 405)),
    ("bf16", "forward", "product", 128, False, (8320, 256, 448)),
    ("bf16", "forward", "product", 128, True, (5540, 6697, 133)),
    ("bf16", "forward", "product", 128, True, (192, 5888, 8448)),
    ("bf16", "forward", "product", 256, False, (780, 203, 9595)),
    ("bf16", "forward", "product", 256, False, (832, 256, 9408)),
    ("bf16", "forward", "product", 256, True, (133, 6601, 8427)),
    ("bf16", "forward", "product", 256, True, (8256, 4160, 448)),
    ("bf16", "dx", "lone", 128, False, (74, 65, 215)),
    ("bf16", "dx", "lone", 128, False, (128, 64, 256)),
    ("bf16", "dx", "lone", 128, True, (69, 71, 641)),
    ("bf16", "dx", "lone", 128, True, (128, 64, 704)),
    ("bf16", "dx", "product", 32, False, (4, 65, 201)),
    ("bf16", "dx", "product", 32, False, (4, 64, 256)),
    ("bf16", "dx", "product", 32, True, (4, 65, 449)),
    ("bf16", "dx", "product", 32, True, (4, 64, 512)),
    ("bf16", "dx", "product", 64, False, (38, 65, 207)),
    ("bf16", "dx", "product", 64, False, (33, 64, 256)),
    ("bf16", "dx", "product", 64, True, (38, 65, 475)),
    ("bf16", "dx", "product", 64, True, (33, 64, 512)),
    ("bf16", "dx", "product", 128, False, (386, 9079, 201)),
    ("bf16", "dx", "product", 128, False, (448, 8320, 256)),
    ("bf16", "dx", "product", 128, True, (5631, 131, 6617)),
    ("bf16", "dx", "product", 128, True, (5440, 192, 8896)),
    ("bf16", "dx", "product", 256, False, (8324, 903, 205)),
    ("bf16", "dx", "product", 256, False, (1088, 7232, 256)),
    ("bf16", "dx", "product", 256, True, (8720, 145, 6549)),
    ("bf16", "dx", "product", 256, True, (8256, 448, 3840)),
    ("bf16", "dw", "lone", 128, False, (206, 65, 65)),
    ("bf16", "dw", "lone", 128, False, (256, 64, 64)),
    ("bf16", "dw", "lone", 128, True, (649, 67, 77)),
    ("bf16", "dw", "lone", 128, True, (704, 64, 64)),
    ("bf16", "dw", "product", 128, False, (202, 9119, 387)),
    ("bf16", "dw", "product", 128, False, (256, 8256, 448)),
    ("bf16", "dw", "product", 128, True, (4717, 8335, 129)),
    ("bf16", "dw", "product", 128, True, (5888, 192, 8448)),
    ("bf16", "dw", "product", 256, False, (201, 9505, 781)),
    ("bf16", "dw", "product", 256, False, (256, 960, 8256)),
    ("bf16", "dw", "product", 256, True, (5777, 143, 8223)),
    ("bf16", "dw", "product", 256, True, (4032, 576, 6592)),
]


def path_of(dtype, which, shape):
    from paper_2504_05638_amd import binding as B
    kernel, tile, parts = B.tagc_linear_path_host(PASSES.index(which), *shape, {"f32": B.TAGC_F32, "bf16": B.TAGC_BF16}[dtype])
    return KERNELS[kernel], tile, parts > 1


@pytest.mark.parametrize("dtype,which,kernel,tile,in_parts,shape", PATHS, ids=lambda v: str(v).replace(" ", ""))
def test_path(dtype, which, kernel, tile, in_parts, shape):
    from paper_2504_05638_amd.train import linear, linear_backward
    print("[case]", dtype, which, kernel, tile, in_parts, shape, flush=True)
    assert path_of(dtype, which, shape) == (kernel, tile, in_parts)
    M, K, N = shape
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M + K + N)
    x, w, dy = (torch.randn(s, generator=gen, device="cuda").to(T[dtype]) for s in ((M, K), (N, K), (M, N)))
    if which == "forward":
        got, p, q = linear(x, w)[0], x.double(), w.double().t()
    elif which == "dx":
        got, p, q = linear_backward(dy, x, w), dy.double(), w.double()
    else:
        got = torch.empty_like(w)
        linear_backward(dy, x, w, dw=got, need_dx=False)
        p, q = dy.double().t(), x.double()
    ref, size = p @ q, p.abs() @ q.abs()
    err = (p.shape[1] + 8) * 2 * E * size
    half = 2.0 ** -8 if dtype == "bf16" else E
    off = (got.double() - ref).abs()
    assert torch.isfinite(got).all()
    assert torch.all(off <= err + half * (ref.abs() + err)), float((off - err).max())
