"""No-GPU checks of study_worker_step.py: a round through which nothing gets ends with an error."""
import pytest
import torch

import study_worker_step as study


class Deaf:
    """An aggregator's calls as Receiver.round makes them; no packet ever counts, and more passes than a limit are refused."""
    n_pkts = 5

    def __init__(self, most):
        self.left = most

    def begin_round(self, number):
        pass

    def packetize(self, *a, **k):
        pass

    def packetize_list(self, *a):
        pass

    def apply_arrivals_queue(self, packets, count, queue):
        pass

    def loss_account(self, bound, missing, names):
        self.left -= 1
        assert self.left >= 0, "sent again without end"
        return 10, False, None


@pytest.mark.parametrize("arrives", [0, 3])
def test_a_round_that_nothing_gets_through_ends(arrives):
    r = study.Receiver.__new__(study.Receiver)
    r.agg, r.workers, r.bound = Deaf(2000), 2, 20_000
    r.packets = r.src = r.missing = None
    r.list = torch.zeros(10, dtype=torch.int64)
    r.of_worker = torch.zeros(10, dtype=torch.int64)
    r.arrivals = lambda of_worker: torch.arange(arrives)
    with pytest.raises(RuntimeError, match="round 7"):
        r.round(7, [None, None])


@pytest.mark.parametrize("loss", [1.0, -0.1, 2.0, float("nan")])
def test_a_loss_of_everything_is_refused(loss):
    with pytest.raises(ValueError):
        study.Receiver(None, 2, loss, 20_000)
