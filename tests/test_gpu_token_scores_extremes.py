"""Token scores of rows that hold very large finite logits, either sign, beside ordinary ones: as masks, as single logits, throughout.
Against 64 bits, within the tolerances of ordinary rows."""
import pytest
import torch

from tests.test_gpu_token_scores import DEV, check, logits, some_tokens

pytestmark = pytest.mark.gpu
# chunks of 256 vectors to a row, and rows: a wave to a row of one chunk and of three, four waves twice, eight, eight or sixteen, sixteen, five parts
WAYS = [(0.7, 0), (2.5, 2048), (2.5, 0), (5.3, 0), (7.9, 0), (18.3, 0), (30.1, 0), (70.2, 0)]
TYPES = [torch.float32, torch.bfloat16]


def length(chunks, dtype):
    return int(chunks * (1024 if dtype == torch.float32 else 2048))


def check_rows(q, x, rows, seed):
    """The rows of x by themselves (in two calls where they are too many to be cut into parts), or among `rows` in all."""
    if rows > x.shape[0]:
        x = x.repeat((rows + x.shape[0] - 1) // x.shape[0], 1)
    for piece in x.split(60) if x.shape[1] > 50000 and not rows else [x]:
        t = some_tokens(seed, piece.shape[0], piece.shape[1])
        t[::2] = piece[::2].float().argmax(dim=1).int()
        for n in (0, 3, 40):
            check(q, piece, t, n)


@pytest.mark.parametrize("chunks,rows", WAYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_large_magnitude(gpu_lib, chunks, rows, dtype):
    """One constant in the tail or the head of a row, as masks are added: exponentials against it may be large and their products with
    exponents larger."""
    V = length(chunks, dtype)
    values = [-1e4, -1e7, -11629081.0, -11629160.0, -1e9, -3080770304.0, -1e10, -1e11, -1e38]
    values += (-3e9 * (20 / 3) ** torch.rand(15, generator=torch.Generator().manual_seed(1))).tolist()
    x = logits(V, 2 * len(values), V, dtype)
    for i, v in enumerate(values):
        x[2 * i, (1, 300, V // 3, V // 8)[i % 4]:] = v
        x[2 * i + 1, :(1, 300, V // 2, V - 2)[i % 4]] = v
    check_rows(gpu_lib, x, rows, 3)


@pytest.mark.parametrize("chunks,rows", WAYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_one_very_large_logit(gpu_lib, chunks, rows, dtype):
    """In what is read first, and later."""
    V = length(chunks, dtype)
    g = torch.Generator().manual_seed(2)
    values = [1.1e7, 11629079.0, 11629081.0, 11629165.0, 1.2e7, 2e9, 5e9, 1e10, 1e11, 1e15, 1e20, 1e30, 3e38]
    values += (1e9 * 20 ** torch.rand(24, generator=g)).tolist() + (1e10 * 2 ** torch.rand(11, generator=g)).tolist()
    x = logits(V, 2 * len(values), V, dtype)
    for i, v in enumerate(values):
        x[2 * i, (5, min(300, V - 1), V // 2 + 3, V - 1)[i % 4]] = v
        x[2 * i + 1, torch.randint(0, V, (1,), generator=g).item()] = v
    check_rows(gpu_lib, x, rows, 4)


@pytest.mark.parametrize("chunks,rows", WAYS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_an_ordinary_logit(gpu_lib, chunks, rows, dtype):
    """One far above the others, all of them large; one and nothing else; all equal; ordinary differences around a large logit."""
    V = length(chunks, dtype)
    base = logits(V, 1, V, torch.float32)[0]
    made = []
    for at in (5, V // 2 + 3, V - 1):
        for high, low in ((-1e10, -2e10), (-1e7, -1e9), (1e10, 0.99e10), (2e9, -2e9), (-1e9, float("-inf")), (1.4e10, float("-inf")), (-1e9, -3e38)):
            r = torch.full((V,), low, device=DEV)
            r[at] = high
            made.append(r)
    for c in [11629079.0 + 4 * i for i in range(25)] + [-11629079.0 - 16 * i for i in range(12)] + [1e10, -1e10, 1e30, -1e30]:
        made += [torch.full((V,), c, device=DEV), torch.full((V,), c, device=DEV) + torch.round(base)]
    check_rows(gpu_lib, torch.stack(made).to(dtype), rows, 5)


@pytest.mark.parametrize("V", [50, 3000, 9001, 100000])
def test_tokens_far_below_the_others(gpu_lib, V):
    """A masked token's log probability is its own logit but for the row's lse, rounded once."""
    rows = 200
    x = logits(V, rows, V, torch.float32)
    t = some_tokens(V, rows, V)
    g = torch.Generator().manual_seed(6)
    low = -torch.exp2(torch.randint(10, 127, (rows,), generator=g)) * (1 + 0.2 * torch.rand(rows, generator=g))
    x[torch.arange(rows, device=DEV), t.long()] = low.to(DEV)
    check(gpu_lib, x, t, 0)
    check(gpu_lib, x[:, :40].contiguous(), t % 40, 40)
