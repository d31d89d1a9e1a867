"""Which sizes the matrix product takes, asked of the library on the CPU through its workspaces."""
import pytest


def layer():
    from paper_2606_16907_amd import layer as L
    L.load_library()
    return L


def forward_bytes(m, n, k):
    """Rows at odd addresses are packed first, which takes a workspace; 0 where the sizes are refused."""
    L = layer()
    a = L.TgLinearArgs(x=4098, w=8194, y=65536, m=m, n=n, k=k, ldx=k, ldw=k, ldy=n, type=1, out_type=1)
    return L.load_library().tg_linear_workspace_bytes(a)


def gradient_bytes(m, n, k):
    L = layer()
    a = L.TgLinearGradArgs(dy=4096, pre=4096, x=8194, w=8194, dx=4096, dw=4096, m=m, n=n, k=k, lddy=n, ldp=n, ldx=k, ldw=k, lddx=k, lddw=k,
                           type=1, act=2)
    return L.load_library().tg_linear_grad_workspace_bytes(a)


LARGE = [(1 << 20, 1 << 15, 64), (1 << 20, 64, 1 << 15), (1 << 24, 2048, 2048), (0x7fffffff - 256, 8, 128), (4096, (1 << 21) - 64, 4096),
         (1 << 16, (1 << 21) - 64, 512)]


@pytest.mark.parametrize("m,n,k", LARGE)
def test_sizes_within_the_limits_are_taken(m, n, k):
    assert forward_bytes(m, n, k) >= (m + n) * k * 2
    assert gradient_bytes(m, n, k) >= m * n * 2


@pytest.mark.parametrize("m,n,k", [(1 << 31, 8, 8), (100, 1 << 21, 8), (100, 8, 1 << 21), (1 << 24, 1 << 14, 8), (1 << 24, 8, 1 << 14),
                                   (8, 1 << 20, 1 << 18)])
def test_sizes_beyond_them_are_not(m, n, k):
    assert forward_bytes(m, n, k) == 0 and gradient_bytes(m, n, k) == 0
