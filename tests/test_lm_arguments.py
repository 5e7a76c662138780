"""What the language-model operators' torch functions hand to the library, checked on the host with a stand-in for it:
pointers, strides and sizes, and what is refused before anything is enqueued."""
import pytest
import torch

from paper_1906_02367_b200 import lm


class Recorder:
    """Takes the place of the library: keeps the arguments of every call and reports success."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 4096 if name == "qs_embed_grad_bytes" else 0
        return call


@pytest.fixture
def calls(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(lm, "lib", lambda: rec)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(lm, "_allocate", lambda stream, shape, dtype, device: torch.zeros(shape, dtype=dtype))
    monkeypatch.setattr(lm, "_handle", lambda stream, device: 0)
    return rec.calls


def operators(status):
    """Every function that takes a status word."""
    tok, table, z, u = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8), torch.zeros(4, 10), torch.zeros(4, 2)
    ids, lse = torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4)
    return [lambda: lm.embed(tok, table, status=status), lambda: lm.embed_grad(tok, torch.zeros(4, 8), 10, status=status),
            lambda: lm.token_logp(z, tok, status=status), lambda: lm.token_logp_grad(z, tok, lse, status=status),
            lambda: lm.distill(z, ids, u, status=status), lambda: lm.distill_grad(z, ids, u, lse, 1.0, status=status)]


@pytest.mark.parametrize("status", [torch.zeros(1, dtype=torch.int8), torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32),
                                    torch.zeros(1, dtype=torch.float32)])
def test_a_status_word_is_one_int32(calls, status):
    """The device writes four bytes there: anything else would be written past its end, or read back as another number."""
    for call in operators(status):
        del calls[:]
        with pytest.raises(ValueError):
            call()
        assert all(name == "qs_embed_grad_bytes" for name, _ in calls)
    for call in operators(torch.zeros(1, dtype=torch.int32)) + operators(torch.zeros((), dtype=torch.int32)):
        call()


def test_a_workspace_is_one_stretch_of_memory(calls):
    """Its size is counted from its elements, so they have to lie side by side: every other byte of a buffer would be
    taken for all of it."""
    tok, go = torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    buf = torch.zeros(8192, dtype=torch.uint8)
    for work in (buf[::2], torch.zeros(1, dtype=torch.uint8).expand(8192), torch.zeros(64, 64).t()):
        with pytest.raises(ValueError):
            lm.embed_grad(tok, go, 10, work=work)
    assert not calls
    lm.embed_grad(tok, go, 10, work=buf)
    lm.embed_grad(tok, go, 10, work=torch.zeros(64, 32))
    assert [c[1][15] for c in calls] == [8192, 8192]


def strides_of(calls, name):
    """(table's worker and row stride, out's row stride) of qs_embed; grad_out's row stride of qs_embed_grad."""
    args = [a for n, a in calls if n == name][-1]
    return (args[8], args[9], args[13]) if name == "qs_embed" else args[8]


def test_dimensions_of_one_element_have_no_stride(calls):
    """The last position of each of several sequences, (B, 1, D) of (B, S, D): rows one sequence apart; and a single row,
    whatever strides its dimensions of one element carry."""
    B, S, D = 3, 5, 8
    hidden, tok, table = torch.zeros(B, S, D), torch.zeros((B, 1), dtype=torch.int64), torch.zeros(10, D)
    lm.embed(tok, table, out=hidden[:, -1:, :])
    assert strides_of(calls, "qs_embed") == (0, D, S * D)
    lm.embed_grad(tok, hidden[:, -1:, :], 10, workers=False)
    assert strides_of(calls, "qs_embed_grad") == S * D
    lm.embed(tok, table, out=torch.as_strided(hidden, (B, 1, D), (S * D, 1, 1)))
    assert strides_of(calls, "qs_embed") == (0, D, S * D)
    lm.embed(tok[:1], table, out=torch.as_strided(hidden, (1, 1, D), (1, 1, 1)))
    assert strides_of(calls, "qs_embed")[2] >= D
    lm.embed_grad(tok[0, 0], hidden[0, 0], 10)           # one token without a dimension
    assert strides_of(calls, "qs_embed_grad") >= D
    lm.embed(torch.zeros((2, 1, 4), dtype=torch.int64), table, out=torch.as_strided(hidden, (2, 1, 4, D), (4 * D, 1, D, 1)))
    assert strides_of(calls, "qs_embed") == (0, D, D)
    z = torch.as_strided(torch.zeros(64), (1, 10), (1, 1))
    lm.token_logp(z, torch.zeros(1, dtype=torch.int64))
    assert calls[-1][1][4] >= 10
    with pytest.raises(ValueError):                      # every other element
        lm.embed(tok, table, out=torch.zeros(B, 1, 2 * D)[..., ::2])
    # expanded dimensions: rows of stride 0 are the library's to refuse, they are not taken for rows side by side
    assert lm._rows(torch.zeros(1, 1, D).expand(2, 3, D), "rows") == 0
    with pytest.raises(ValueError):
        lm._rows(torch.zeros(2, 1, D).expand(2, 3, D), "rows")
    with pytest.raises(ValueError):                      # rows whose two dimensions do not flatten
        lm.embed(torch.zeros((2, 2), dtype=torch.int64), table, out=torch.zeros(2, 3, D)[:, :2])


def test_tiles_of_a_long_list_are_few():
    """Every tile of the sort reads the counts of all tiles: their number has a bound, up to the most tokens that are taken.
    The workspace shows it: 16 bytes a token, the partial sums of chunks of 64, and the rest."""
    from paper_1906_02367_b200 import binding as B
    L = B.lib()
    for R, N in ((1, 1 << 30), (1, 20_000_000), (32, 1 << 25), (8, 3_000_000)):
        chunks = R * (N // 64 + 1)
        rest = L.qs_embed_grad_bytes(R, N, 128000, 1) - 16 * R * N - chunks * (2 * 256 * 4 + 4) - R * 128000
        assert rest <= 2 * R * 2048 * 512 * 4 + 1024, (R, N, rest)


def test_strides_of_rows_address_the_same_elements():
    """Whatever stride is taken for a tensor of any shape and strides, the rows found with it are the tensor's."""
    g, base, taken = torch.Generator().manual_seed(3), torch.arange(4000), 0
    pick = lambda values: values[int(torch.randint(0, len(values), (1,), generator=g))]  # noqa: E731
    for _ in range(3000):
        dims = pick((1, 2, 3, 4))
        shape, stride = [pick((1, 1, 2, 3)) for _ in range(dims)], [pick((0, 1, 2, 3, 4, 6, 9, 12, 18)) for _ in range(dims)]
        stride[-1] = pick((1, 1, stride[-1]))
        t = torch.as_strided(base, shape, stride)
        try:
            step = lm._rows(t, "rows")
        except ValueError:
            continue
        flat = t.reshape(-1, shape[-1])
        assert torch.equal(flat, torch.stack([base[i * step:i * step + shape[-1]] for i in range(len(flat))])), (shape, stride, step)
        taken += 1
    assert taken > 1000
