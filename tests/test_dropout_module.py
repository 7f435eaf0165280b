"""The Dropout module under recomputation, in processes that train together and in
copies of a network (CPU, the kernel replaced by the generator on the host), and
recomputation on the kernel (needs an MI355X)."""

from __future__ import annotations

import copy
import os
import socket

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import torch.distributed as dist  # noqa: E402
import torch.multiprocessing as mp  # noqa: E402
from torch.utils.checkpoint import checkpoint  # noqa: E402

import paper_2301_03251_amd as Q  # noqa: E402
from paper_2301_03251_amd import drop  # noqa: E402
from test_dropout import philox  # noqa: E402

MODES = [False, True]  # checkpoint's use_reentrant


def on_host(x, p, key):
    """``dropout_forward`` of CPU tensors."""
    seed, offset = (int(k) % (1 << 64) for k in key)
    n = x.numel()
    words = philox(np.arange((n + 3) // 4, dtype=np.uint64), offset, seed).reshape(-1)[:n]
    keep = torch.from_numpy(words.astype(np.int64) >= round(p * 2.0 ** 32)).view(x.shape)
    return torch.where(keep, x / (1 - p), torch.zeros_like(x))


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(drop, "dropout_forward", on_host)


class Net(torch.nn.Module):
    """Two dropouts, the first one also called twice; what is around them needs its inputs again."""

    def __init__(self, device="cpu"):
        super().__init__()
        torch.manual_seed(1)
        self.a, self.b = torch.nn.Linear(12, 16, device=device), torch.nn.Linear(16, 5, device=device)
        self.first, self.second = Q.Dropout(0.4, seed=3, device=device), Q.Dropout(0.2, seed=4, device=device)

    def forward(self, x, keys=(None, None, None)):
        y = self.first(torch.tanh(self.a(x)), keys[0])
        return self.second(torch.tanh(self.b(torch.sin(self.first(y * y, keys[1])))), keys[2])

    def draw(self):
        return self.first.draw(), self.first.draw(), self.second.draw()


def gradients(net, loss):
    return torch.autograd.grad(loss, list(net.parameters()))


def recomputed(device):
    x = torch.randn(9, 12, device=device)
    for reentrant in MODES:
        x = x.detach().requires_grad_(reentrant)
        plain, net = Net(device), Net(device)
        for _ in range(2):  # the second step goes on from the first one's counters
            want = gradients(plain, plain(x).square().sum())
            keys = net.draw()
            y = checkpoint(lambda x, *k: net(x, k), x, *keys, use_reentrant=reentrant)
            if reentrant:  # takes gradients by .backward() alone
                net.zero_grad()
                y.square().sum().backward()
                got = [p.grad for p in net.parameters()]
            else:
                got = gradients(net, y.square().sum())
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert torch.equal(net.first.key, plain.first.key) and net.first.key.tolist() == [3, 4]


def refused(device):
    """Each mode, whichever layers are inside; neither counts a call that was refused."""
    x = torch.randn(9, 12, device=device, requires_grad=True)
    for reentrant in MODES:
        net = Net(device)
        y = checkpoint(net, x, use_reentrant=reentrant)
        assert net.first.key.tolist() == [3, 2] and net.second.key.tolist() == [4, 1]
        with pytest.raises(RuntimeError, match="backward pass"):
            y.sum().backward()
        assert net.first.key.tolist() == [3, 2] and net.second.key.tolist() == [4, 1]
        # what drops nothing may be run again
        net.eval()
        checkpoint(net, x, use_reentrant=reentrant).sum().backward()


def test_recomputation(host):
    """Keys drawn outside give the gradients of the network without recomputation."""
    recomputed("cpu")


def test_recomputation_without_keys_is_refused(host):
    """A mask of its own in the second forward pass would give another function's gradients."""
    refused("cpu")


def test_draw(host):
    layer, x = Q.Dropout(0.5, seed=8, device="cpu"), torch.randn(30, 7)
    keys = [layer.draw() for _ in range(3)]
    assert [k.tolist() for k in keys] == [[8, 0], [8, 1], [8, 2]] and layer.key.tolist() == [8, 3]
    assert torch.equal(layer(x, keys[1]), on_host(x, 0.5, (8, 1))) and layer.key.tolist() == [8, 3]
    assert torch.equal(layer(x, (8, 1)), on_host(x, 0.5, (8, 1)))
    assert torch.equal(layer(x), on_host(x, 0.5, (8, 3))) and layer.key.tolist() == [8, 4]


def _rank(rank, port, path):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port), RANK=str(rank), WORLD_SIZE="2")
    dist.init_process_group("gloo")
    drop.dropout_forward = on_host
    torch.manual_seed(0)
    net = torch.nn.Sequential(torch.nn.Linear(6, 40), Q.Dropout(0.5, seed=100 + rank, device="cpu"))
    both = torch.nn.parallel.DistributedDataParallel(net)
    masks = []
    for _ in range(3):
        y = both(torch.ones(8, 6))
        masks.append(y.detach() != 0)
        y.sum().backward()
    torch.save((net[1].key.clone(), torch.stack(masks)), f"{path}/{rank}")
    dist.destroy_process_group()


def test_processes_keep_their_seeds(tmp_path):
    """DistributedDataParallel makes the ranks' parameters and buffers alike, but not their masks."""
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    mp.spawn(_rank, (port, str(tmp_path)), nprocs=2)
    (a, m), (b, n) = (torch.load(tmp_path / str(r), weights_only=True) for r in range(2))
    assert a.tolist() == [100, 3] and b.tolist() == [101, 3]
    assert all((m[i] != n[i]).any() for i in range(3))


def test_copies_have_masks_of_their_own(host):
    """Blocks of a network that are copies of one, as layers with seeds of their own."""
    block = torch.nn.Sequential(torch.nn.Linear(6, 40), Q.Dropout(0.5, seed=9, device="cpu"))
    block[1].draw()
    torch.manual_seed(5)
    first, second = copy.deepcopy(block), copy.deepcopy(block)
    assert block[1].key.tolist() == [9, 1]
    keys = [m[1].key.tolist() for m in (block, first, second)]
    assert len({k[0] for k in keys}) == 3 and keys[1][1] == keys[2][1] == 0
    x = torch.ones(8, 6)
    masks = [m(x) != 0 for m in (block, first, second)]
    assert (masks[0] != masks[1]).any() and (masks[0] != masks[2]).any() and (masks[1] != masks[2]).any()
    assert torch.equal(first[0].weight, block[0].weight) and first[1].p == 0.5 and first[1].training
    torch.manual_seed(5)
    assert copy.deepcopy(block)[1].key.tolist() == keys[1]
    # one layer in two places is one layer in the copy too
    shared = torch.nn.ModuleList([block[1], block[1]])
    twin = copy.deepcopy(shared)
    assert twin[0] is twin[1] and twin[0] is not block[1]


def test_state(host):
    """The key is part of the state under its name, follows the module, and a loaded one keeps its address."""
    net = torch.nn.Sequential(Q.Dropout(0.5, seed=9, device="cpu"))
    net[0].draw()
    state = net.state_dict()
    assert list(state) == ["0.key"] and state["0.key"].tolist() == [9, 1]
    other = torch.nn.Sequential(Q.Dropout(0.5, device="cpu"))
    held = other[0].key
    assert str(other.load_state_dict(state)) == "<All keys matched successfully>"
    assert other[0].key is held and held.tolist() == [9, 1]
    state["0.key"].zero_()
    assert held.tolist() == [9, 1]
    assert other.load_state_dict({}, strict=False).missing_keys == ["0.key"]
    with pytest.raises(RuntimeError, match="Missing key"):
        other.load_state_dict({})
    with pytest.raises(RuntimeError, match="size mismatch"):
        other.load_state_dict({"0.key": torch.zeros(3, dtype=torch.int64)})
    assert other.half().double()[0].key.dtype == torch.int64
    assert other.to("meta")[0].key.device.type == "meta"
    other.load_state_dict({"0.key": torch.tensor([2, 6])}, assign=True)
    assert other[0].key.tolist() == [2, 6]


def test_a_key_of_numbers_is_kept_as_it_was(host):
    """The gradient's mask is the forward's, whatever becomes of the caller's list."""
    key, x = [3, 4], torch.randn(40, 5, requires_grad=True)
    y = Q.dropout(x, 0.5, key)
    key[1] = 5
    y.sum().backward()
    assert torch.equal(x.grad, on_host(torch.ones_like(x), 0.5, (3, 4)))


@pytest.mark.gpu
def test_recomputation_on_the_kernel():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    recomputed("cuda")
    refused("cuda")
