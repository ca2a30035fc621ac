// What the translation unit of the language-model operators shares with the rest of the library.
#pragma once

namespace ifq {

// Read and clear that unit's device status word on the current device (an ifq_status: IFQ_OK or
// IFQ_ECUDA where the read failed).  The caller has synchronised.
int lm_take_status(int* status);

}  // namespace ifq
