"""Device memory that the head loss takes, against what the header states."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")

MIB = 1 << 20


def _taken(T, D, V):
    """MiB that a first loss and gradient of T tokens allocates, and the call's results and arguments."""
    g = torch.Generator(device="cuda").manual_seed(T + D)
    W = torch.empty(V, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(2.0 * D ** -0.5)
    X = torch.empty(T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    dloss = torch.ones(T, device="cuda")
    out = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(X)
    h = pkg.Handle()
    h.sq_head_loss_grad(X[:1, :64].contiguous(), W[:64, :64].contiguous(), labels[:1] % 64, dloss[:1])  # kernels are loaded
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    h.sq_head_loss_grad(X, W, labels, dloss, *out)
    h.sq_sync()
    return (free - torch.cuda.mem_get_info()[0]) / MIB, out, (X, W, labels)


@pytest.mark.parametrize("T, D, V, most", [
    # 16 rows of exponentials of 4 MiB and their sums, where 256 would take 1 GiB
    (1, 8, 1 << 21, 16 * 4 * 1.1 + 64),
    # planes of 64 MiB, of which 19 would be the fastest; 256 packed rows
    (1, 65536, 128256, 512 + 32 + 64),
    # 9216 rows: packed 1152 MiB, planes in chunks of 2048 where all together take 2304 MiB
    (9000, 65536, 512, 1152 + 512 + 64),
    # the exponentials of 2048 rows a chunk, planes of 32 MiB
    (3000, 4096, 128256, 24 + 1.1 * 512 + 512),
])
def test_scratch_of_a_gradient(T, D, V, most):
    torch.cuda.empty_cache()
    taken, (loss, lse, dX), (X, W, labels) = _taken(T, D, V)
    assert taken <= most
    for t in sorted({0, T // 2, T - 1}):
        z = torch.cat([(w.double() @ X[t].double()) for w in W.split(16384)])
        assert abs(float(lse[t]) - float(torch.logsumexp(z, 0))) < 1e-3
        p = torch.softmax(z, 0)
        p[labels[t]] -= 1
        want = sum(p[i:i + 16384] @ W[i:i + 16384].double() for i in range(0, V, 16384))
        assert float((dX[t].double() - want).norm() / want.norm()) <= 1.25 * 2.0 ** -8
