"""Host-only checks of the training operators: what their workspaces come to, and what they refuse, without touching a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2509_11254_b200 import binding, build

    build.build_library()
    return binding.lib()


def size(L, call, *args):
    n = C.c_size_t(1 << 62)
    assert getattr(L, call)(*args, C.byref(n)) == 0
    return n.value


def test_loss_workspace_holds_no_logits(L):
    for T, V in ((1, 32000), (777, 50257), (16384, 131072)):
        # 8 bytes per 128 logits (statistics), 4 + 2 bytes per token and alignment
        assert size(L, "psgd_xent_workspace", T, V, 768, 0) <= T * (8 * (V // 128 + 1) + 16) + 4096


def test_gradient_workspace_is_bounded_in_tokens(L):
    """16 bits per logit of at most 2^29 logits at a time, statistics (1/8 byte per logit), float32 sums of the weight gradient once there
    are several pieces, and partial tiles of products that are cut along their contraction."""
    V, D = 131072, 1024
    one = size(L, "psgd_xent_workspace", 4096, V, D, 1)
    many = [size(L, "psgd_xent_workspace", T, V, D, 1) for T in (8192, 65536, 1 << 20)]
    tiles = 4096 * 65536 * 4          # generous: partial tiles of both products
    for T, n in zip((8192, 65536, 1 << 20), many):
        assert n <= (1 << 29) * 17 // 8 + V * D * 4 + T * 16 + tiles + (1 << 20)
    assert one <= 4096 * (V * 17 // 8) + 4096 * 16 + tiles + (1 << 20)
    assert many[2] - many[1] <= ((1 << 20) - 65536) * 16 + tiles      # growing with tokens only by the loss's per-row terms
    # a small vocabulary needs no pieces for a long time
    assert size(L, "psgd_xent_workspace", 1 << 17, 1000, 64, 1) < 1 << 30


def test_weight_gradient_workspace(L):
    # a bfloat16 form of the checkpoint and partial tiles
    assert size(L, "psgd_act_wgrad_workspace", 4096, 2048, 768) <= 4096 * 768 * 2 + 256 * 65536 * 4 + 4096
    assert size(L, "psgd_act_wgrad_workspace", 0, 2048, 768) > 0


def test_queries_refuse(L):
    n = C.c_size_t()
    for bad in ((-1, 10, 10), (10, 0, 10), (10, 10, 0), (1 << 31, 10, 10), (10, 1 << 31, 10), (10, 10, 1 << 31)):
        assert L.psgd_xent_workspace(*bad, 1, C.byref(n)) == -1
        assert L.psgd_act_wgrad_workspace(bad[0], bad[1], bad[2], C.byref(n)) == -1
    assert L.psgd_xent_workspace(8, 8, 8, 1, None) == -2 and L.psgd_act_wgrad_workspace(8, 8, 8, None) == -2


def test_calls_refuse_before_any_launch(L):
    p = 1 << 20          # stands for device addresses; nothing below gets as far as using one
    xent = lambda T=8, V=16, D=64, H=p, ldh=64, W=p, ldw=64, lab=p, loss=p, ws=p, nb=1 << 40: L.psgd_xent_loss(
        H, ldh, W, ldw, lab, None, -100, T, V, D, loss, p, p, None, ws, nb, None)
    assert xent(H=None) == -2 and xent(W=None) == -2 and xent(lab=None) == -2 and xent(loss=None) == -2 and xent(ws=None) == -2
    assert xent(H=p + 8) == -1 and xent(W=p + 2) == -1 and xent(ldh=63) == -1 and xent(ldw=65) == -1 and xent(ws=p + 8) == -1
    assert xent(T=-1) == -1 and xent(V=0) == -1 and xent(D=0) == -1 and xent(nb=0) == -3
    assert L.psgd_act_pack(p, 64, 1, -1, 64, p, p, None) == -1 and L.psgd_act_pack(p, 64, 1, 8, 0, p, p, None) == -1
    assert L.psgd_act_pack(p, 64, 7, 8, 64, p, p, None) == -1 and L.psgd_act_pack(p, 64, 1, 8, 64, p, None, None) == -2
    assert L.psgd_act_pack(p, 64, 1, 0, 64, None, None, None) == 0
    assert L.psgd_act_unpack(p + 4, p, 8, 64, p, 64, 0, None) == -1 and L.psgd_act_unpack(p, p, 8, 64, p, 63, 0, None) == -1
    assert L.psgd_act_wgrad(p, 16, p, p, 8, 16, 64, p, 63, 0, None, p, 1 << 40, None) == -1
    assert L.psgd_act_wgrad(p, 16, p, p, 8, 16, 64, p, 64, 0, None, p, 0, None) == -3
    assert L.psgd_act_wgrad(p + 8, 16, p, p, 8, 16, 64, p, 64, 0, None, p, 1 << 40, None) == -1
    assert L.psgd_swiglu_forward(p, 64, p, 64, 8, 64, p, 63, p, p, p, p, None) == -1 and L.psgd_swiglu_forward(p, 64, None, 64, 8, 64, p, 64, p, p, p, p, None) == -2
    assert L.psgd_swiglu_backward(p, 64, p, p, p, p, 8, 64, p, 64, p, 64, p, 10, None) == -1


def test_copy_rows_refuses(L):
    p = 1 << 20
    assert L.psgd_copy_rows(p, 7, 4, 8, p, 8, None) == -1 and L.psgd_copy_rows(p, 8, 4, 8, p, 7, None) == -1 and L.psgd_copy_rows(p, 8, -1, 8, p, 8, None) == -1
    assert L.psgd_copy_rows(None, 8, 4, 8, p, 8, None) == -2 and L.psgd_copy_rows(None, 8, 0, 8, None, 8, None) == 0


def test_python_refuses_host_tensors():
    import torch

    import paper_2509_11254_b200 as p

    h, w, y = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: p.linear_cross_entropy(h, w, y), lambda: p.linear_cross_entropy_grad(h, w, y), lambda: p.pack_activation(h), lambda: p.swiglu_forward(h, h),
                 lambda: p.weight_gradient(h, None), lambda: p.swiglu_backward(h, None, None)):
        with pytest.raises(p.PSGDError):
            call()


def test_overlapping_outputs_are_refused(L):
    """Outputs that share a byte with an operand or with each other are refused; rows that only lie between one another's (columns of one wider matrix) are not.
    Placements at random against sets of bytes; the workspace is too small (-3) wherever the arguments pass, so that nothing is launched."""
    import random

    rng = random.Random(1)
    p = 1 << 20

    def cells(at, rows, cols, ld, size):
        return {at + r * ld * size + b for r in range(rows) for b in range(cols * size)}

    seen = {-1: 0, -3: 0}
    for _ in range(4000):
        T, V, D = rng.choice([1, 2, 3, 7]), rng.choice([1, 2, 5, 9]), rng.choice([8, 24])
        ld = [D + 8 * rng.randrange(6) for _ in range(2)] + [D + rng.randrange(40) for _ in range(2)]
        if rng.random() < 0.6:
            ld = [rng.choice([64, 72])] * 4                             # columns of one buffer
        at = [p + 16 * rng.randrange(40) * rng.choice([0, 1, 4, 16]) for _ in range(2)] + [p + 2 * rng.randrange(320) * rng.choice([0, 1, 4, 16]) for _ in range(2)]
        h, w, dh, dw = (cells(a, n, D, s, 2) for a, n, s in zip(at, (T, V, T, V), ld))
        want = -1 if dh & h or dh & w or dw & h or dw & w or dh & dw else -3
        got = L.psgd_xent_grad(at[0], ld[0], at[1], ld[1], p, None, -100, T, V, D, p, p, p, at[2], ld[2], at[3], ld[3], None, p, 0, None)
        assert got == want, (T, V, D, at, ld)
        seen[got] += 1
    assert min(seen.values()) > 400
    import torch

    if torch.cuda.is_available():           # (the addresses are made up: where there is a GPU, only calls that end at the workspace's size are made)
        return
    for size, dw in ((4, p), (2, p + 2 * 7), (4, p + 5 * 48 - 8)):         # dY: 6 rows of 16, 24 apart
        assert L.psgd_act_wgrad(p, 24, p, p, 6, 16, 9, dw, 24, 0 if size == 4 else 1, None, p, 1 << 40, None) == -1


def test_loss_workspace_is_bounded_in_tokens(L):
    """Statistics (8 bytes per 128 logits) of at most 2^25 x 128 logits at a time, and 16 bytes per 8 tokens; never more than the gradients need."""
    for V in (32000, 131072):
        for T in (1 << 17, 1 << 20, 1 << 24):
            n = size(L, "psgd_xent_workspace", T, V, 2048, 0)
            assert n <= (1 << 28) + (1 << 25) // (V // 128) * 4 + 2 * T + 4096
            assert n <= size(L, "psgd_xent_workspace", T, V, 2048, 1)


def test_failed_launch_says_why(L):
    """Without a GPU every launch fails: the exception carries the runtime's text, and it is this thread's."""
    import threading

    import torch

    from paper_2509_11254_b200 import PSGDError, training

    if torch.cuda.is_available():
        pytest.skip("the address below is made up")
    p = 1 << 20
    code = L.psgd_act_pack(p, 64, 1, 8, 64, p, p, None)
    assert code == -4
    with pytest.raises(PSGDError, match="PSGD_E_CUDA: kernel launch: .*(device|driver)"):
        training._check(code)
    other = []
    t = threading.Thread(target=lambda: other.append(L.psgd_training_cuda_error()))
    t.start()
    t.join()
    assert other == [b"no error"]


def test_stream_of_another_device_is_refused():
    """(It would make its own device current, on which the call would never find itself at home.)"""
    import types

    import torch

    from paper_2509_11254_b200 import PSGDError, training

    stream = types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    with pytest.raises(PSGDError, match="stream is on cuda:1"):
        with training._there(torch.device("cuda", 0), stream):
            pass
