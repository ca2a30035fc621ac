// What the translation units of the language-model operators share with the rest of the library.
#pragma once

namespace ifq {

// Read and clear a unit's device status word on the current device (an ifq_status: IFQ_OK or
// IFQ_ECUDA where the read failed).  The caller has synchronised.
int lm_take_status(int* status);      // the attention block's
int layer_take_status(int* status);   // the rest of a layer's, and the scores'

}  // namespace ifq
