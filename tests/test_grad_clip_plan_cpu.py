"""What a GradientClip's plan points to: memory that stays there as long as the object does, and whether it is still where a program's gradients are.
CPU tensors: a plan is laid down without a GPU."""
import torch
from torch.multiprocessing.reductions import StorageWeakRef

import paper_2508_06001_amd as K


def gradients():
    return [torch.ones((5, 3)), torch.ones((7,), dtype=torch.bfloat16), torch.empty((0,)), torch.ones((2, 8, 2))]


def test_the_memory_of_a_plan_outlives_tensors_that_are_given_other_memory():
    grads = gradients()
    out = [g.clone() for g in grads]
    c = K.GradientClip(grads, 1.0, out=out)
    kept = [StorageWeakRef(t.untyped_storage()) for t in (grads[0], out[1])]
    grads[0].data = torch.zeros((5, 3))
    out[1].data = torch.zeros((7,), dtype=torch.bfloat16)
    assert not any(k.expired() for k in kept)
    del c
    assert all(k.expired() for k in kept)


def test_a_list_of_other_gradients_is_told_apart():
    grads = gradients()
    c = K.GradientClip(grads, 1.0)
    assert c.stands_for(grads) and c.stands_for(iter(grads)) and c.stands_for([g.view(-1) for g in grads])
    assert not c.stands_for(grads[:-1]) and not c.stands_for(grads[::-1]) and not c.stands_for(gradients())      # as a step leaves them that frees its gradients
    assert not c.stands_for([grads[0][:4]] + grads[1:]) and not c.stands_for([grads[0].view(torch.int32)] + grads[1:])
    assert not c.stands_for([None] + grads[1:])
    grads[3].data = torch.ones((2, 8, 2))
    assert not c.stands_for(grads)
    out = gradients()
    c = K.GradientClip(gradients(), 1.0, out=out)
    assert c.stands_for(c.grads) and not c.stands_for(out)
