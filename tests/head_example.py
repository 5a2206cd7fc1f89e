"""The example of a head on a state, as the README has it."""

EXAMPLE = """\
from paper_2508_06993_amd.runtime import CellLayer, Dropout
cells = state[..., 0].numel()
new = lambda *shape: torch.zeros(*shape, device="cuda")
layers = [CellLayer(torch.randn(48, 16, device="cuda"), new(48), rows=cells, train=True),
          CellLayer(torch.randn(19, 48, device="cuda"), new(19), rows=cells, train=True)]
drop, pre, hidden, scores = Dropout(0.1, seed=1), new(cells, 48), new(cells, 48), new(cells, 19)
layers[0].forward(state, pre)
drop(pre, hidden, gate=pre)                            # ReLU and dropout
layers[1].forward(hidden, scores)
grad_scores, grad_hidden, grad_state = scores, new(cells, 48), new(cells, 16)   # of 1/2 scores^2
layers[1].backward(grad_scores, grad_hidden)           # fills grad_weight, grad_bias
drop(grad_hidden, grad_hidden, gate=pre)               # the same call on the gradient
layers[0].backward(grad_hidden, grad_state)
"""
