"""What the Python binding checks before it hands addresses to the library (no GPU needed: handles of no device,
tensors on the CPU)."""
import pytest
import torch

import paper_1907_09356_b200 as choco


def embedding(n, vocab, dim, row=0, ld=0):
    h = choco.EmbeddingHandle()
    h.describe(-1, n, vocab, dim, row, ld)
    return h


@pytest.mark.parametrize("layout,shape,strides,good", [
    ((3, 10, 4), (3, 40), (40, 1), True), ((3, 10, 4), (4, 50), (40, 1), True),
    ((3, 10, 4), (3, 39), (40, 1), False),                       # a table's last row ends behind its row of X
    ((3, 10, 4), (2, 40), (40, 1), False),                       # too few workers
    ((3, 10, 4), (3, 40), (41, 1), False), ((3, 10, 4), (3, 40), (0, 1), False),   # another pitch than the handle's
    ((3, 10, 4), (3, 40), (1, 3), False),                        # columns apart
    ((3, 10, 4, 0, 55), (3, 40), (55, 1), True), ((3, 10, 4, 0, 55), (3, 55), (54, 1), False),
    ((3, 10, 4, 6, 70), (3, 58), (70, 1), True), ((3, 10, 4, 6, 70), (3, 57), (70, 1), False),
    ((3, 10, 4), (3, 10, 4), (40, 4, 1), True), ((3, 10, 4), (3, 10, 4), (40, 5, 1), False),
    ((3, 10, 4), (3, 9, 4), (40, 4, 1), False), ((3, 10, 4), (3, 10, 3), (40, 4, 1), False), ((3, 10, 4), (3, 10, 4), (40, 1, 10), False),
    ((3, 10, 4), (120,), (1,), True), ((3, 10, 4), (119,), (1,), False), ((3, 10, 4), (120,), (2,), False),
    ((1, 10, 4), (1, 40), (7, 1), True), ((1, 10, 4), (10, 4), (4, 1), True), ((1, 10, 4), (10, 4), (5, 1), False),
    ((1, 10, 4, 6), (10, 4), (6, 1), True), ((1, 10, 4), (9, 4), (4, 1), False), ((1, 10, 4), (40,), (1,), True),
    ((3, 10, 4), (), (), False), ((3, 10, 4), (1, 3, 10, 4), (120, 40, 4, 1), False)])
def test_tables_hold_what_the_handle_describes(layout, shape, strides, good):
    t = torch.zeros(400).as_strided(shape, strides)
    h = embedding(*layout)
    if good:
        choco._check_table(h, "a table", t)
    else:
        with pytest.raises(choco.ChocoError, match="does not hold"):
            choco._check_table(h, "a table", t)


def test_lookup_and_gradient_look_at_table_and_device_before_the_call(monkeypatch):
    def no_call():
        raise AssertionError("the library was called")
    monkeypatch.setattr(choco, "load", no_call)
    h = embedding(2, 10, 4)
    tok, rows, X = torch.zeros((2, 3), dtype=torch.int64), torch.zeros((2, 3, 4)), torch.zeros((2, 40))
    for call in (lambda: choco.choco_embedding_forward(h, X[:, :39], tok, rows), lambda: choco.choco_embedding_backward(h, tok, rows, X[:, 1:])):
        with pytest.raises(choco.ChocoError, match="does not hold"):
            call()
    for bad_tok, bad_rows in ((tok[:1], rows[:1]), (tok, rows[:, :2]), (tok, rows[:, :, :3])):   # of fewer workers than the handle's
        with pytest.raises(choco.ChocoError, match="tokens must be"):
            choco.choco_embedding_forward(h, X, bad_tok, bad_rows)
    with pytest.raises(choco.ChocoError, match="the handle is for"):
        choco.choco_embedding_forward(h, X, tok[:1], rows[:1], n=1)
    h.device = 1                                                 # the tensors are elsewhere
    for call in (lambda: choco.choco_embedding_forward(h, X, tok, rows), lambda: choco.choco_embedding_backward(h, tok, rows, X)):
        with pytest.raises(choco.ChocoError, match="on one GPU"):
            call()
    h.device = -1
    with pytest.raises(AssertionError):                          # and with everything in place it goes on
        choco.choco_embedding_forward(h, X, tok, rows)


def test_handles_pass_as_pointers():
    import ctypes
    libc = ctypes.CDLL(None)
    libc.strlen.argtypes, libc.strlen.restype = [ctypes.c_void_p], ctypes.c_size_t
    text = ctypes.create_string_buffer(b"five.")
    h = choco.EmbeddingHandle(ctypes.addressof(text))
    assert libc.strlen(h) == 5
    libc.memcpy.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, ctypes.c_size_t]
    word = ctypes.c_uint64(0x1234)
    libc.memcpy(ctypes.byref(h), ctypes.addressof(word), 8)      # as an init call writes it
    assert h.value == 0x1234


def adamw(n_tensors=6, groups=3, bits=32, elements=1024):
    h = choco.AdamWHandle()
    h.describe(-1, n_tensors, groups, bits, elements)
    return h


@pytest.fixture
def no_library(monkeypatch):
    def no_call():
        raise AssertionError("the library was called")
    monkeypatch.setattr(choco, "load", no_call)


def refused(call, match):
    with pytest.raises(choco.ChocoError, match=match):
        call()


@pytest.mark.parametrize("bad", [torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.bfloat16), torch.zeros(2), torch.zeros(6)[::2]])
def test_norms_and_factors_are_one_float_per_group(no_library, bad):
    h, fine = adamw(), torch.zeros(3)
    m = torch.zeros(1024)
    message = "one element for each of 3 groups|are not supported"
    refused(lambda: choco.choco_adamw_grad_norm(h, 1.0, bad, fine), message)
    refused(lambda: choco.choco_adamw_grad_norm(h, 1.0, fine, bad), message)
    refused(lambda: choco.choco_adamw_step(h, m, m.clone(), None, None, 1e-3, bad), message)
    h.device = 1
    refused(lambda: choco.choco_adamw_grad_norm(h, 1.0, fine, fine), message)


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_are_those_of_the_list(no_library, bits):
    h, factor = adamw(bits=bits), torch.zeros(3)
    make = lambda kinds: [torch.zeros(c, dtype=getattr(torch, k)) for k, c in kinds]  # noqa: E731
    fine = make(h.state_arrays())
    assert [a.numel() for a in fine] == ([1024, 1024] if bits == 32 else [1024, 1024, 4, 4])
    padded = lambda a: (list(a) + [None, None])[:4]  # noqa: E731
    wrong = []
    for k in range(len(fine)):
        wrong += [fine[:k] + [a] + fine[k + 1:] for a in (None, fine[k][:-1], fine[k].double(), torch.zeros(2 * len(fine[k]), dtype=fine[k].dtype)[::2])]
    for states in wrong:
        refused(lambda: choco.choco_adamw_step(h, *padded(states), 1e-3, factor), "the moments must be")
        if all(a is not None for a in states):
            refused(lambda: choco.choco_adamw_read_state(h, *padded(states), torch.zeros(1024), None), "the moments must be")
    for out in (torch.zeros(1023), torch.zeros(2048)[::2]):
        refused(lambda: choco.choco_adamw_read_state(h, *padded(fine), out, None), "outputs must be")
    with pytest.raises(AssertionError):                          # all in place: it goes on, for one output alone too
        choco.choco_adamw_step(h, *padded(fine), 1e-3, None)
    only_m = [a if k % 2 == 0 else None for k, a in enumerate(padded(fine))]
    with pytest.raises(AssertionError):
        choco.choco_adamw_read_state(h, *only_m, torch.zeros(1024), None)
    h.device = 1
    refused(lambda: choco.choco_adamw_step(h, *padded(fine), 1e-3, None), "the moments must be")


def test_host_arrays_have_an_element_for_each_tensor_or_group(no_library):
    h = adamw()
    refused(lambda: choco.choco_adamw_state_size(h, 5), "6 tensors")
    refused(lambda: choco.choco_adamw_set_grads(h, [4096] * 5), "6 tensors")
    refused(lambda: choco.choco_adamw_set_grads(h, [[4096] * 6]), "6 tensors")
    refused(lambda: choco.choco_adamw_get_steps(h, 2), "3 groups")
    refused(lambda: choco.choco_adamw_set_steps(h, [1, 2]), "3 groups")
    refused(lambda: choco.choco_adamw_set_steps(h, 1), "3 groups")


def test_rows_of_one_list_are_on_one_gpu():
    class Elsewhere:                                             # a tensor of another GPU, as far as the checks look
        is_cuda, shape, device = True, (2, 10), "cuda:1"

        def get_device(self):
            return 1

        def dim(self):
            return 2

        def stride(self, k):
            return (10, 1)[k]

    class Here(Elsewhere):
        device = "cuda:0"

        def get_device(self):
            return 0

    refused(lambda: choco.adamw_layer_tensors(Elsewhere(), Here(), [0, 10]), "G on cuda:0")
